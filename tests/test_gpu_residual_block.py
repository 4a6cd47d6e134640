"""Norm, gated layer, layer and dropout together, as a residual block uses them: against plain torch in 64 bits, in a
captured graph, in the example, and one after the other on other streams."""
import os
import sys

import pytest
import torch

import plain_layers
from paper_2410_22697_amd import (AdamW, RowFormat, dropout, dropout_backward, gated, gated_backward, linear, linear_backward, rms_norm,
                                  rms_norm_backward, unpack_rows)

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu
EPS = 1e-6


def parameters(width, hidden, dtype=torch.float32, seed=0):
    g = torch.Generator().manual_seed(seed)
    new = lambda *s: torch.randn(s, generator=g).div_(s[-1] ** 0.5 if len(s) > 1 else 4).cuda().to(dtype)  # noqa: E731
    return [1 + new(width), new(2 * hidden, width), new(2 * hidden), new(width, hidden), new(width)]


def block(h, p, seed, draw):
    scale, both, bias, back, end = p
    return dropout(linear(gated(rms_norm(h, scale, EPS), both, bias), back, end), 0.3, seed, draw, residual=h)


def plain_block(h, p, seed, draw):
    scale, both, bias, back, end = p
    n = both.shape[0] // 2
    z = (h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * scale) @ both.t() + bias
    y = torch.nn.functional.silu(z[:, :n]) * z[:, n:]
    keep = torch.from_numpy(plain_layers.kept(*h.shape, 0.3, seed, draw)).cuda()
    return h + torch.where(keep, (y @ back.t() + end) / 0.7, 0.0)


@pytest.mark.parametrize("rows,width,hidden", [(7, 24, 40), (300, 64, 128), (5000, 33, 70)])
def test_two_blocks_against_plain_torch(rows, width, hidden):
    """fp32: a result is a chain of some ten sums of a few hundred terms, each rounded once a term; they come out 1e-5 of their
    size off at the very most, in norm far below."""
    ps = [[t.requires_grad_() for t in parameters(width, hidden, seed=i)] for i in range(2)]
    x, v = torch.randn(rows, width, device="cuda", requires_grad=True), torch.randn(rows, width, device="cuda")
    y = block(block(x, ps[0], 5, 0), ps[1], 5, 1)
    y.backward(v)
    qs = [[t.detach().double().requires_grad_() for t in p] for p in ps]
    xd = x.detach().double().requires_grad_()
    want = plain_block(plain_block(xd, qs[0], 5, 0), qs[1], 5, 1)
    want.backward(v.double())
    assert (y - want).norm() <= 1e-5 * want.norm()
    for t, q in zip([x, *ps[0], *ps[1]], [xd, *qs[0], *qs[1]]):
        assert (t.grad - q.grad).norm() <= 1e-5 * q.grad.norm()


def test_a_step_replayed():
    """Forward, backward and the optimizer's step as calls of their own, the seed in memory, and the normed rows packed."""
    rows, width, hidden = 2100, 128, 256
    scale, both, bias, back, end = p = parameters(width, hidden, torch.bfloat16)
    start = [t.clone() for t in p]
    x, dy = (torch.empty(rows, width, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    seed, fmt, opt = torch.zeros(1, dtype=torch.int64, device="cuda"), RowFormat(width, 8), AdamW(p, state_bits=8)

    def step():
        n = rms_norm(x, scale, EPS)
        y, pre = gated(n, both, bias, save_pre=True)
        out = dropout(linear(y, back, end), 0.3, seed, 1, residual=x)
        dz = dropout_backward(dy, 0.3, seed, 1)
        d, _, dback, dend = linear_backward(dz, y, back)
        dn, _, dboth, dbias = gated_backward(d, n, both, pre)
        dx, dscale = rms_norm_backward(dn, x, scale, EPS, ds=dy)
        opt.t = 0
        opt.step([dscale, dboth, dbias, dback, dend])
        table, total = rms_norm(out, scale, EPS, residual=x, fmt=fmt)
        seed.add_(1)
        return out, dx, table, total, unpack_rows(table, fmt)

    def fresh(at):
        g = torch.Generator(device="cuda").manual_seed(at)
        for t in (x, dy):
            t.copy_(torch.randn(rows, width, device="cuda", generator=g))
        for t, s in zip(p, start):
            t.copy_(s)
        for t in (opt.m, opt.v, opt.m_scale, opt.v_scale):
            t.zero_()
        seed.fill_(at)

    fresh(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for at in (3, 4, 3, 9):
        fresh(at)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, *p, *opt.states())]
        fresh(at)
        want = [*step(), *p, *opt.states()]
        torch.cuda.synchronize()
        for i, (u, v) in enumerate(zip(got, want)):
            assert torch.equal(u, v), (at, i)
        assert int(seed) == at + 1


def test_two_graphs_and_eager_calls_side_by_side():
    """Two captured backward passes, replayed on two streams at once, beside the eager one."""
    rows, width, hidden = 3000, 64, 200
    p = parameters(width, hidden)
    xs = [torch.randn(rows, width, device="cuda") for _ in range(2)]
    dys = [torch.randn(rows, hidden, device="cuda") for _ in range(2)]

    def grads(i):
        y, pre = gated(xs[i], p[1], p[2], save_pre=True)
        return (y, *gated_backward(dys[i], xs[i], p[1], pre), *rms_norm_backward(xs[1 - i], xs[i], p[0], EPS))

    want = [[t for t in grads(i) if t is not None] for i in range(2)]
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for i in range(2):
        streams[i].wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(streams[i]):
            grads(i)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            outs.append([t for t in grads(i) if t is not None])
    torch.cuda.synchronize()
    for _ in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        here = [[t for t in grads(i) if t is not None] for i in range(2)]
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(u, v) and torch.equal(u, w) for u, v, w in zip(want[i], outs[i], here[i]))


def test_the_example_with_blocks():
    from train_sage import Setup, train
    s = Setup(8, width=96, blocks=2, drop=0.0)
    seeds, packed, blocks = s.sample(0)
    loss = torch.nn.functional.cross_entropy(s.logits(packed, blocks), s.labels[seeds.long()])
    loss.backward()
    own = [p.grad.clone() for p in s.params]
    assert all(torch.isfinite(g).all() and g.any() for g in own)
    losses = train(6, report=None, blocks=1)
    assert torch.isfinite(losses).all()
