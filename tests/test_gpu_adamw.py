"""The AdamW step: parameters and 32-bit states against the formula in 64 bits, 8-bit states code for code against the
formula's fp32 steps."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import AdamW

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
SIZES = [1, 3, 255, 256, 257, 1000, 4096, 4099, 20_000]


def cpu(t):
    return t.detach().float().cpu().numpy().reshape(-1)


def check_params(new, old, g, m, v, t, dtype):
    """new against the 64-bit step from fp32 states. A moment's error is two roundings of each of its terms, the update's
    its quotient's few; sqrt(v) halves v's error."""
    b1, b2 = HYPER["betas"]
    want, m64, v64 = plain.adamw(old, g, m, v, t, HYPER["lr"], b1, b2, HYPER["eps"], HYPER["weight_decay"])
    terms = b1 * np.abs(m) + (1 - b1) * np.abs(g)
    denom = np.sqrt(v64) / np.sqrt(1 - b2 ** t) + HYPER["eps"]
    rate = HYPER["lr"] / (1 - b1 ** t)
    slack = rate * (4 * terms + 12 * np.abs(m64)) * plain.EPS / denom + 4 * plain.EPS * np.abs(old) + 1e-30
    half = plain.BF / 2 * (np.abs(want) + slack) if dtype == torch.bfloat16 else 0.0
    assert np.all(np.abs(new.astype(np.float64) - want) <= slack + half)
    return m64, v64, terms


def make(sizes, param, grad, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    params = [torch.randn(n, generator=g, device="cuda").to(param) for n in sizes]
    grads = lambda: [(torch.randn(n, generator=g, device="cuda") * torch.rand(n, generator=g, device="cuda").square()).to(grad) for n in sizes]  # noqa: E731
    return params, grads


@pytest.mark.parametrize("param", ["f32", "bf16"])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("bits", [32, 8])
def test_steps(param, grad, bits):
    params, grads = make(SIZES, TYPES[param], TYPES[grad])
    copies = [torch.empty_like(p, dtype=torch.bfloat16) if i % 2 else None for i, p in enumerate(params)]
    opt = AdamW(params, state_bits=bits, copies=copies, **HYPER)
    for t in (1, 2, 3):
        g = grads()
        old = [cpu(p) for p in params]
        m0, v0 = (cpu(s).copy() for s in opt.states())
        opt.step(g)
        m1, v1 = (cpu(s) for s in opt.states())
        for i, (p, a) in enumerate(zip(params, opt.starts)):
            n = p.numel()
            m, v, gi = m0[a:a + n], v0[a:a + n], cpu(g[i])
            m64, v64, terms = check_params(cpu(p), old[i], gi, m, v, t, p.dtype)
            m32, v32 = plain.moments32(gi, m, v, *HYPER["betas"])
            if bits == 32:
                assert np.all(np.abs(m1[a:a + n] - m64) <= 3 * plain.EPS * terms)
                assert np.all(np.abs(v1[a:a + n] - v64) <= 4 * plain.EPS * v64)
            else:
                cm, sm = plain.encode(m32, 2)
                cv, sv = plain.encode(v32, 4)
                blocks = slice(a // 256, a // 256 + len(sm))
                assert np.array_equal(opt.m[a:a + n].cpu().numpy(), cm) and np.array_equal(opt.v[a:a + n].cpu().numpy(), cv)
                assert np.array_equal(opt.m_scale[blocks].cpu().numpy(), sm)
                assert np.array_equal(opt.v_scale[blocks].cpu().numpy(), sv)
                assert np.array_equal(m1[a:a + n], plain.decode(cm, sm, 2)) and np.array_equal(v1[a:a + n], plain.decode(cv, sv, 4))
                # what a code stands for: half a code's width off at most, in the root
                top = np.repeat(np.abs(plain.blocks(m32)).max(1), 256)[:n]
                assert np.all(np.abs(np.sqrt(np.abs(m1[a:a + n])) - np.sqrt(np.abs(m32))) <= np.sqrt(top) * (0.5 / 127 + 1e-6))
            rest = slice(a + n, a + -(-n // 256) * 256)
            assert np.all(m1[rest] == 0) and np.all(v1[rest] == 0)
            if copies[i] is not None:
                assert torch.equal(copies[i], p.to(torch.bfloat16))
    assert opt.t == 3


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_holds_and_odd_addresses(bits):
    """130 tensors, views that begin anywhere in a larger array; what lies between them stays."""
    sizes = [1 + (37 * i) % 700 for i in range(130)]
    flat, gflat = torch.randn(sum(sizes) + 3 * 131, device="cuda"), torch.randn(sum(sizes) + 131, device="cuda")
    at, gat, params, grads, between = 3, 1, [], [], []
    for n in sizes:
        params.append(flat[at:at + n])
        between += [at + n, at + n + 1, at + n + 2]
        grads.append(gflat[gat:gat + n])
        at, gat = at + n + 3, gat + n + 1
    before = flat.clone()
    opt = AdamW(params, state_bits=bits, **HYPER)
    opt.step(grads)
    old = before.cpu().numpy()
    at = 3
    for p, g in zip(params, grads):
        n = p.numel()
        zero = np.zeros(n, np.float32)
        check_params(cpu(p), old[at:at + n], cpu(g), zero, zero, 1, torch.float32)
        at += n + 3
    keep = torch.tensor([i for i in [0, 1, 2] + between if i < flat.numel()], device="cuda")
    assert torch.equal(flat[keep], before[keep])


def test_gradients_from_autograd_and_missing_ones():
    params, _ = make([300, 70], torch.float32, torch.float32)
    for p in params:
        p.requires_grad_()
    opt = AdamW(params, **HYPER)
    opt.step()  # no gradient at all: no step
    assert opt.t == 0
    (params[0] * torch.linspace(-1, 1, 300, device="cuda")).sum().backward()
    old = [cpu(p).copy() for p in params]
    opt.step()
    assert opt.t == 1 and np.array_equal(cpu(params[1]), old[1])
    zero = np.zeros(300, np.float32)
    check_params(cpu(params[0]), old[0], cpu(params[0].grad), zero, zero, 1, torch.float32)


def test_values_that_are_not_finite_stay_in_their_block():
    params, _ = make([1024], torch.float32, torch.float32)
    g = torch.randn(1024, device="cuda")
    g[300], g[600] = float("nan"), float("inf")
    opt = AdamW(params, state_bits=8, **HYPER)
    opt.step([g])
    m, v = (s.cpu().numpy() for s in opt.states())
    for block in (0, 3):
        assert np.isfinite(m[block * 256:block * 256 + 256]).all() and np.isfinite(v[block * 256:block * 256 + 256]).all()
    for block in (1, 2):
        assert np.isnan(m[block * 256:block * 256 + 256]).all() and np.isnan(v[block * 256:block * 256 + 256]).all()
    # the parameter of a finite gradient took its step with the 32-bit moments
    assert torch.isfinite(params[0][:300]).all() and torch.isnan(params[0][300])


def test_small_and_zero_gradients():
    """Blocks under a scale's reach hold zeros, and a step with them is finite; without gradient only the decay acts."""
    params, _ = make([512], torch.float32, torch.float32)
    old = cpu(params[0]).copy()
    g = torch.zeros(512, device="cuda")
    g[256:] = 2.0 ** -130
    opt = AdamW(params, state_bits=8, **HYPER)
    opt.step([g])
    assert torch.all(opt.m == 0) and torch.all(opt.v == 0) and torch.all(opt.m_scale == 0) and torch.all(opt.v_scale == 0)
    assert np.allclose(cpu(params[0]), old * (1 - HYPER["lr"] * HYPER["weight_decay"]), rtol=2e-7)


def test_tiny_v_next_to_a_large_one_is_not_held_as_zero():
    """A code of 0 for v > 0 would divide by eps alone on the next step."""
    params, _ = make([256], torch.float32, torch.float32)
    g = torch.full((256,), 1e-6, device="cuda")
    g[0] = 10.0
    opt = AdamW(params, state_bits=8, **HYPER)
    before = params[0].clone()
    for _ in range(20):
        opt.step([g])
    assert torch.all(opt.v[1:] >= 1)
    assert (params[0] - before).abs().max() < 20 * HYPER["lr"] * 3


@pytest.mark.parametrize("n", [1, 2, 3, 5, 255, 257, 1030])
def test_states_of_any_length(n):
    """The library call takes lengths that are no multiple of four; Python's arrays are padded to 256."""
    import ctypes
    from paper_2410_22697_amd import operators
    lib = operators._load()
    rng = np.random.default_rng(n)
    cm, cv = rng.integers(-127, 128, n).astype(np.int8), rng.integers(0, 256, n).astype(np.uint8)
    sm, sv = rng.random((2, -(-n // 256))).astype(np.float32)
    d = [torch.from_numpy(x).cuda() for x in (cm, cv, sm, sv)]
    m, v = (torch.full((n + 4,), 5.0, device="cuda") for _ in range(2))
    rc = lib.massive_adamw_states(*(t.data_ptr() for t in d), n, m.data_ptr(), v.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0, ctypes.string_at(lib.massive_last_error(None))
    assert np.array_equal(m[:n].cpu().numpy(), plain.decode(cm.astype(np.int64), sm, 2))
    assert np.array_equal(v[:n].cpu().numpy(), plain.decode(cv.astype(np.int64), sv, 4))
    assert torch.all(m[n:] == 5) and torch.all(v[n:] == 5)


def test_refusals():
    p, g = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    for bad in (lambda: AdamW([]), lambda: AdamW([p.half()]), lambda: AdamW([p, p.bfloat16()]), lambda: AdamW([p[::2]]),
                lambda: AdamW([p.cpu()]), lambda: AdamW([p], state_bits=16), lambda: AdamW([p], copies=[p]),
                lambda: AdamW([p], copies=[]), lambda: AdamW([p]).step([]), lambda: AdamW([p]).step([g[:4]]),
                lambda: AdamW([p]).step([g.cpu()]), lambda: AdamW([p]).step([g.half()]),
                lambda: AdamW([p, p]).step([g, g.bfloat16()])):
        with pytest.raises(ValueError):
            bad()
    from paper_2410_22697_amd import MassiveError
    for wrong in (dict(lr=-1.0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=float("nan")), dict(weight_decay=-1.0)):
        opt = AdamW([p], **wrong)
        with pytest.raises(MassiveError):
            opt.step([g])
        assert opt.t == 0
