"""One block of a text encoder as a program uses the calls together: token lookup, norm, 8-bit integer projection, norm with gate and residual, their gradients, and the update of
everything with AdamW; eager, in a graph, on two streams, and for single tokens."""
import numpy as np
import pytest
import torch

import paper_2211_12281_amd as kge

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
V, D, SEQ, LEN = 400, 256, 6, 40                 # tokens of the vocabulary, width, sequences of so many positions
EPS = 1e-5
NAMES = ["pre.w", "pre.b", "post.w", "post.b", "last.w", "last.b", "scale"]


def _values(shape, *key, std=1.0, mean=0.0):
    return torch.from_numpy(np.random.default_rng([int(k) for k in key]).normal(size=shape) * std + mean).float()


class Block:
    """Parameters, moments and the step; nothing is kept between steps but these."""

    def __init__(self, bits=8):
        vec = lambda i, m: _values(D, 1, i, std=0.2, mean=m).cuda()                                    # noqa: E731
        self.p = {"table": _values((V, D), 2).cuda(), "w": _values((D, D), 3, std=D ** -0.5).cuda()}
        self.p |= {n: vec(i, 1.0 if n.endswith("w") else 0.5 if n == "scale" else 0.0) for i, n in enumerate(NAMES)}
        self.shadow = {n: self.p[n].to(BF16) if n in ("table", "w") else None for n in self.p}
        self.opt = kge.AdamW(self.p.values(), shadows=self.shadow.values(), bits=[bits if t.dim() == 2 else 32 for t in self.p.values()],
                             weight_decay=[0.01 if t.dim() == 2 else 0.0 for t in self.p.values()], seed=99)
        self.spaces = [kge.Workspace() for _ in range(7)]
        for s in self.spaces:
            s.get(32 << 20)

    def norm(self, name):
        return kge.Norm("layer", self.p[name + ".w"], self.p[name + ".b"], EPS)

    def forward(self, ids, gate, ws=None, stream=None):
        pre, post, last = (self.norm(n) for n in ("pre", "post", "last"))
        x = kge.embed(self.shadow["table"], ids, dtype=F32, stream=stream)
        _, z = kge.norm_block(x, pre=pre, dtype=BF16, stream=stream)
        wq = kge.quantize_rowwise(self.shadow["w"], by="both", stream=stream, ws=ws and ws[0])
        y = kge.matmul_rowwise(kge.quantize_rowwise(z, stream=stream), wq[0], stream=stream, ws=ws and ws[1])
        h, out = kge.norm_block(x, y, post=post, pre=last, scale=self.p["scale"], gate=gate, gate_rows=LEN, stream=stream)
        return x, z, wq, y, h, out

    def step(self, ids, gate, dout, step, ws=None, counter=None, stream=None):
        """(output, gradients); the parameters after the update are self.p"""
        k = ws or [None] * 7
        x, z, wq, y, h, out = self.forward(ids, gate, ws, stream)
        g = kge.norm_block_bwd(h, y, dz=dout, post=self.norm("post"), pre=self.norm("last"), scale=self.p["scale"], gate=gate, gate_rows=LEN, ws=k[2], stream=stream)
        dy_row, dy_col = kge.quantize_rowwise(g["y"], by="both", ws=k[3], stream=stream)
        dz = kge.matmul_rowwise(dy_row, wq[1], ws=k[1], stream=stream)
        dw = kge.matmul_rowwise(dy_col, kge.quantize_rowwise(z, by="col", ws=k[0], stream=stream), dtype=F32, ws=k[4], stream=stream)
        first = kge.norm_block_bwd(x, dh=g["x"], dz=dz, pre=self.norm("pre"), ws=k[5], stream=stream)
        dt = kge.embed_bwd(first["x"], ids, V, ws=k[6], stream=stream)
        grads = dict(table=dt, w=dw, scale=g["scale"])
        grads |= {"pre.w": first["pre_weight"], "pre.b": first["pre_bias"], "post.w": g["post_weight"], "post.b": g["post_bias"],
                  "last.w": g["pre_weight"], "last.b": g["pre_bias"]}
        self.opt.step([grads[n] for n in self.p], 1e-2, step, step_counter=counter, stream=stream)
        return dict(out=out, gate=g["gate"], **grads)

    def state(self):
        return [*self.p.values(), *(s for s in self.shadow.values() if s is not None), *(t for s in self.opt.states for t in (s.m, s.v))]


def _inputs(key=0):
    ids = torch.from_numpy(np.random.default_rng([5, key]).integers(0, V, size=SEQ * LEN).astype(np.int32))
    ids[7], ids[-1] = -1, -1
    return ids.cuda(), _values((SEQ, D), 6, key).to(BF16).cuda(), _values((SEQ * LEN, D), 7, key, std=0.1).to(BF16).cuda()


def test_a_training_step():
    """Against 64 bits without quantisation.  A row of 256 normal values keeps each to half a step of amax / 127, 0.9 % of its root mean square (amax 3.9 of it at most in
    1e4 rows): 1.3 % for a product of two, 2 % through two of them, 0.4 % for each rounding to bf16."""
    b = Block()
    old = {n: t.double().cpu() for n, t in b.p.items()}
    ids, gate, dout = _inputs()
    got = b.step(ids, gate, dout, 1)
    p = {n: (t.to(BF16).double() if n in ("table", "w") else t).requires_grad_() for n, t in old.items()}
    g64 = gate.double().cpu().requires_grad_()
    live = ids.cpu() >= 0
    norm = lambda t, n: torch.nn.functional.layer_norm(t, (D,), p[n + ".w"], p[n + ".b"], EPS)             # noqa: E731
    x = p["table"][ids.cpu().long().clamp(min=0)] * live.unsqueeze(1)
    y = norm(x, "pre") @ p["w"].t()
    out = norm(x + p["scale"] * g64.repeat_interleave(LEN, 0) * norm(y, "post"), "last")
    out.backward(dout.double().cpu())
    want = {"out": out.detach(), "gate": g64.grad, **{n: t.grad for n, t in p.items()}}
    for n, t in want.items():
        err = float((got[n].double().cpu() - t).norm() / t.norm())
        assert err < 0.03, (n, err)
    # the update: AdamW's first step from zero moments moves every element with a gradient by lr, and decays matrices
    for n, t in b.p.items():
        g = got[n].double().cpu()
        move = t.double().cpu() - old[n] * (1 - (1e-2 * 0.01 if t.dim() == 2 else 0.0))
        big = g.abs() > 1e-6
        assert bool(((move + 1e-2 * g.sign())[big].abs() <= 1e-2 * 1e-8 / 1e-6 + 2.0 ** -22 * (old[n][big].abs() + 1e-2)).all()), n
        assert bool((move[g == 0].abs() <= 2.0 ** -23 * old[n][g == 0].abs()).all()), n
        if b.shadow[n] is not None:
            assert torch.equal(b.shadow[n], t.to(BF16))


def test_steps_in_a_graph_with_a_device_counter():
    a, b = Block(), Block()
    ids, gate, dout = _inputs()
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = b.step(ids, gate, dout, 1, ws=b.spaces, counter=counter)
        kge.step_counter_add(counter)
    for i in range(4):
        new = _inputs(i)
        for t, s in zip((ids, gate, dout), new):
            t.copy_(s)
        want = a.step(*new, 1 + i)
        graph.replay()
        torch.cuda.synchronize()
        for n in want:
            assert torch.equal(out[n], want[n]), (i, n)
        for s, t in zip(a.state(), b.state()):
            assert torch.equal(s, t), i


def test_two_streams_at_once_and_the_stream_argument():
    want = []
    for key in range(2):
        b = Block()
        want.append((b, [b.step(*_inputs(key), 1 + i) for i in range(3)]))
    torch.cuda.synchronize()
    blocks, streams, got = [Block() for _ in range(2)], [torch.cuda.Stream() for _ in range(2)], [[], []]
    inputs = [_inputs(key) for key in range(2)]
    torch.cuda.synchronize()
    for i in range(3):
        for key in range(2):
            if key == 0:
                got[0].append(blocks[0].step(*inputs[0], 1 + i, stream=streams[0]))
            else:
                with torch.cuda.stream(streams[1]):
                    got[1].append(blocks[1].step(*inputs[1], 1 + i))
    torch.cuda.synchronize()
    for key in range(2):
        for x, y in zip(want[key][1], got[key]):
            for n in x:
                assert torch.equal(x[n], y[n]), (key, n)
        for s, t in zip(want[key][0].state(), blocks[key].state()):
            assert torch.equal(s, t), key


def test_single_tokens_are_the_rows_of_a_batch():
    """Serving: every position by itself gives what it gives in the batch (sums of integers are exact, a row's norm is summed in one order)."""
    b = Block()
    ids, gate, _ = _inputs()
    out = b.forward(ids, gate)[-1]
    for i in (0, 7, 41, SEQ * LEN - 1):
        one = b.forward(ids[i:i + 1].contiguous(), gate[i // LEN:i // LEN + 1])[-1]
        assert torch.equal(one[0], out[i]), i
