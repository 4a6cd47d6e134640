"""The operators in a captured graph: replays with new inputs and the program's own work between them give what the
eager calls give."""
import pytest
import torch

from paper_2410_22697_amd import (AdamW, RowFormat, block_mean, block_mean_backward, linear, linear_backward, pack_rows, unpack_rows)

pytestmark = pytest.mark.gpu


def test_a_step_replayed():
    rows, n, d, width = 3000, 1200, 64, 96
    fmt = RowFormat(d, 8)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, d, device="cuda")
    table = torch.zeros(rows, fmt.row_bytes, dtype=torch.uint8, device="cuda")
    slots = torch.randperm(rows, generator=gen, device="cuda").to(torch.int32)
    indptr = torch.arange(0, 4 * n + 1, 4, dtype=torch.int32, device="cuda")
    indices = torch.randint(0, rows, (4 * n,), generator=gen, device="cuda", dtype=torch.int32)
    w, b = torch.randn(width, 2 * d, generator=gen, device="cuda") * 0.1, torch.zeros(width, device="cuda")
    start = (w.clone(), b.clone())
    opt = AdamW([w, b], state_bits=8)

    def step():
        pack_rows(x, fmt, out=table, slots=slots)
        own = unpack_rows(table, fmt, index=slots[:n])
        mean = block_mean(table, indptr, indices, fmt=fmt)
        y, pre = linear(own, w, b, act="gelu", x2=mean, save_pre=True)
        dx, dx2, dw, db = linear_backward(y, own, w, "gelu", pre, mean)
        grad = block_mean_backward(dx2, indptr, indices, rows, add=dx)
        opt.t = 0  # the step's number is an argument of the call, which a graph keeps
        opt.step([dw, db])
        return y, dx, dw, db, grad

    def fresh(seed):
        x.copy_(torch.randn(rows, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        w.copy_(start[0])
        b.copy_(start[1])
        for s in (opt.m, opt.v, opt.m_scale, opt.v_scale):
            s.zero_()

    fresh(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for seed in (3, 4, 3, 5):
        fresh(seed)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, w, b, *opt.states())]
        fresh(seed)
        want = [*step(), w, b, *opt.states()]
        torch.cuda.synchronize()
        for i, (u, v) in enumerate(zip(got, want)):
            assert torch.equal(u, v), (seed, i)
