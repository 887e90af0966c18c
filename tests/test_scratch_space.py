"""Scratch space of calls that are given none: calls that run at once - two host threads on torch's default stream, whose launches may alternate -
never hold the same memory, and it belongs to the stream that the kernels run on.  Decided on the host: the library is a stand-in that
notes what it is handed, memory comes from the CPU."""
import contextlib
import threading
import types

import pytest
import torch

import paper_2211_12281_amd.binding as b


class Streams:
    """Stands for torch.cuda.stream: notes the stream that is current in each thread."""

    def __init__(self):
        self.local = threading.local()

    @property
    def current(self):
        return getattr(self.local, "stream", None)

    @contextlib.contextmanager
    def __call__(self, stream):
        before, self.local.stream = self.current, stream
        yield
        self.local.stream = before


class Library:
    """Notes address and size of the scratch space of every call, which returns when `together` calls are in."""

    def __init__(self, together):
        self.gate, self.seen, self.lock = threading.Barrier(together, timeout=20), [], threading.Lock()

    def __getattr__(self, name):
        if name.endswith("workspace_bytes"):
            return lambda *a: 3 << 20

        def call(*args):
            at = [i for i, x in enumerate(args) if isinstance(x, int) and x >= 3 << 20 and (args[i + 1:i + 2] or [None])[0] == 3 << 20]
            assert len(at) == 1, (name, args)
            with self.lock:
                self.seen.append((args[at[0]], args[at[0] + 1]))
            self.gate.wait()
            return 0
        return call


@pytest.fixture
def on_the_host(monkeypatch):
    streams, owner, real = Streams(), {}, torch.empty

    def empty(*a, **k):
        t = real(*a, **{**k, "device": "cpu"})
        owner[t.data_ptr()] = streams.current
        return t
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "stream", streams)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(b, "_here", lambda *t: 0)
    monkeypatch.setattr(b, "_queue", lambda dev, stream: stream.cuda_stream if stream else 7)
    monkeypatch.setattr(b, "_embed_bwd_bytes", lambda *a: 3 << 20)
    monkeypatch.setattr(b, "_matmul_bytes", lambda *a: 3 << 20)
    return owner


class FakeStream:
    cuda_stream = 11


def _embed_bwd(ws=None, stream=None):
    b.embed_bwd(torch.zeros((5, 8)), torch.zeros(5, dtype=torch.int32), 9, ws=ws, stream=stream)


def _matmul(ws=None, stream=None):
    q = b.Quantized(torch.zeros((5, 128), dtype=torch.uint8), torch.zeros((5, 4), dtype=torch.uint8), 100)
    b.matmul_quantized(q, q, ws=ws, stream=stream)


def _at_once(monkeypatch, calls):
    lib = Library(len(calls))
    monkeypatch.setattr(b, "load", lambda: lib)
    errors = []

    def run(c):
        try:
            c()
        except Exception as e:      # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=run, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    return lib.seen


@pytest.mark.parametrize("calls", [(_embed_bwd, _embed_bwd), (_matmul, _matmul), (_embed_bwd, _matmul)])
def test_text_calls_of_two_threads_hold_memory_of_their_own(monkeypatch, on_the_host, calls):
    for _ in range(2):                                       # (the second time with what the first one left behind)
        (p, n), (q, m) = _at_once(monkeypatch, calls)
        assert p + n <= q or q + m <= p


@pytest.mark.parametrize("call", [_embed_bwd, _matmul])
def test_text_calls_take_memory_of_the_stream_they_run_on(monkeypatch, on_the_host, call):
    for stream in (None, FakeStream()):
        ((p, _),) = _at_once(monkeypatch, [lambda: call(stream=stream)])
        assert on_the_host[p] is stream


@pytest.mark.parametrize("call", [_embed_bwd, _matmul])
def test_a_given_workspace_is_used(monkeypatch, on_the_host, call):
    ws = b.Workspace()
    ((p, n),) = _at_once(monkeypatch, [lambda: call(ws=ws)])
    assert (p, n) == (ws.buf.data_ptr(), ws.buf.numel())


# ---------------------------------------------------------------------------------------------
# the path's calls
# ---------------------------------------------------------------------------------------------
def _ids(n):
    return torch.zeros(n, dtype=torch.int32)


def _model():
    m = object.__new__(b.Model)
    m.struct, m.dim, m.rel, m.relw = b.KgeModelT(), 8, torch.zeros((3, 8)), None
    return m


def _score(ws=None):
    b.score(_model(), _ids(4), _ids(4), _ids(4), _ids(6), ws=ws)


def _loss_bwd(ws=None, stream=None):
    b.loss_bwd(_model(), "logsigmoid", _ids(4), _ids(4), _ids(4), _ids(6), ws=ws, stream=stream)


def _sparse_adam(ws=None):
    b.sparse_adam(torch.zeros((9, 8)), None, torch.zeros((9, 8)), torch.zeros((9, 8)), _ids(4), torch.zeros((4, 8)), 0.1, ws=ws)


def _topk(ws=None):
    b.topk(_model(), _ids(4), _ids(4), 0, 9, 2, ws=ws)


def _partition(ws=None):
    b.partition_triples(_ids(4), _ids(4), 3, 2, ws=ws)


def _sampler(ws=None):
    b.TripleSampler(_ids(4), _ids(4), _ids(4), 3, 2, 3, ws=ws)


def _encoder():
    e = object.__new__(b.Encoder)
    e.ref, e.ent_s, e.dim, e.feat_dim = b.KgeEncoderT(), torch.zeros((9, 8)), 8, 16
    return e


def _encode(ws=None):
    _encoder().encode(_ids(4), _ids(4), _ids(6), ws=ws)


def _encode_bwd(ws=None):
    _encoder().encode_bwd(_ids(4), _ids(4), _ids(6), torch.zeros((14, 8)), torch.zeros((14, 8)), ws=ws)


PATH = [_score, _loss_bwd, _sparse_adam, _topk, _partition, _sampler, _encode, _encode_bwd]


@pytest.fixture
def path_on_the_host(monkeypatch, on_the_host):
    monkeypatch.setattr(b, "_i32", lambda t: t)
    monkeypatch.setattr(b, "_stream", lambda stream=None: stream.cuda_stream if stream else 7)
    return on_the_host


@pytest.mark.parametrize("call", PATH)
def test_calls_of_two_threads_hold_memory_of_their_own(monkeypatch, path_on_the_host, call):
    for other in (call, _embed_bwd, _score):
        (p, n), (q, m) = _at_once(monkeypatch, [call, other])
        assert p + n <= q or q + m <= p


@pytest.mark.parametrize("call", PATH)
def test_a_workspace_given_to_the_path_is_used(monkeypatch, path_on_the_host, call):
    ws = b.Workspace()
    ((p, n),) = _at_once(monkeypatch, [lambda: call(ws=ws)])
    assert (p, n) == (ws.buf.data_ptr(), ws.buf.numel())


def test_loss_bwd_takes_memory_of_the_stream_it_runs_on(monkeypatch, path_on_the_host):
    stream = FakeStream()
    ((p, _),) = _at_once(monkeypatch, [lambda: _loss_bwd(stream=stream)])
    assert path_on_the_host[p] is stream


@pytest.mark.parametrize("stream", [None, FakeStream()])
def test_outputs_belong_to_the_stream_that_writes_them(monkeypatch, path_on_the_host, stream):
    calls = [lambda: [b.sample_negatives(1, 2, 3, 0, 9, 5, stream=stream)],
             lambda: [b.sample_negatives_dev(1, None, 2, 3, 0, 9, 5, stream=stream)],
             lambda: list(filter(torch.is_tensor, b.loss_bwd(_model(), "logsigmoid", _ids(4), _ids(4), _ids(4), _ids(6), stream=stream).values()))]
    monkeypatch.setattr(b, "load", lambda: type("Lib", (), {"__getattr__": lambda self, name: lambda *a: 3 << 20 if name.endswith("bytes") else 0})())
    for call in calls:
        for t in call():
            assert path_on_the_host[t.data_ptr()] is stream


@pytest.mark.parametrize("stream", [None, FakeStream()])
def test_a_plan_s_workspace_grows_on_the_stream_that_sorts_into_it(monkeypatch, path_on_the_host, stream):
    t = torch.zeros((9, 8))
    neg = types.SimpleNamespace(numel=lambda: 6, is_cuda=True, dtype=torch.int32, is_contiguous=lambda: True, data_ptr=lambda: 1 << 20)
    calls = [lambda ws: b.sparse_adam_plan(9, 8, _ids(4), ws, stream=stream),
             lambda ws: b.sparse_adam_plan_tables([(9, 8, _ids(4), ws)], stream=stream),
             lambda ws: b.sparse_adam_apply(t, None, t, t, torch.zeros((4, 8)), ws, 0.1, stream=stream),
             lambda ws: b.sparse_adam_apply_tables([(t, None, t, t, torch.zeros((4, 8)), ws)], 0.1, stream=stream),
             lambda ws: b.loss_bwd(_model(), "logsigmoid", _ids(4), _ids(4), _ids(4), neg, draw=(1, 2, 3, 0, 9), plans=[(9, 8, _ids(14), ws)], stream=stream)]
    monkeypatch.setattr(b, "load", lambda: type("Lib", (), {"__getattr__": lambda self, name: lambda *a: 3 << 20 if name.endswith("bytes") else 0})())
    for call in calls:
        ws = b.Workspace()
        call(ws)
        assert path_on_the_host[ws.buf.data_ptr()] is stream
