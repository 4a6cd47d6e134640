"""Tensors that the operators change in place: autograd notices."""
import pytest
import torch

from paper_2410_22697_amd import AdamW, RowFormat, linear, pack_rows, unpack_rows

pytestmark = pytest.mark.gpu
CHANGED = "modified by an inplace operation"


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_between_forward_and_backward_is_noticed(bits):
    w = torch.randn(8, 8, device="cuda", requires_grad=True)
    x = torch.randn(5, 8, device="cuda", requires_grad=True)
    opt = AdamW([w], state_bits=bits)
    y = linear(x, w)
    y.sum().backward(retain_graph=True)
    before = w._version
    opt.step()
    assert w._version > before
    with pytest.raises(RuntimeError, match=CHANGED):
        y.sum().backward()


def test_only_what_a_step_changes_counts_as_changed():
    p, q = (torch.randn(300, device="cuda") for _ in range(2))
    c, d = (torch.zeros(300, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    opt = AdamW([p, q], copies=[c, d])
    g = torch.randn(300, device="cuda")
    was = [t._version for t in (p, q, c, d, g)]
    m, v = opt.states()
    held = m._version, v._version
    opt.step([g, None])
    now = [t._version for t in (p, q, c, d, g)]
    assert [a < b for a, b in zip(was, now)] == [True, False, True, False, False]
    assert m._version > held[0] and v._version > held[1]  # 32-bit states are what states() gives


def test_tables_and_outputs_written_to_count_as_changed():
    fmt = RowFormat(16, 8)
    x = torch.randn(4, 16, device="cuda")
    table = pack_rows(x, fmt)
    out = torch.zeros(4, 16, device="cuda")
    was = table._version, out._version
    pack_rows(x, fmt, out=table)
    unpack_rows(table, fmt, out=out)
    assert table._version > was[0] and out._version > was[1]
    a = torch.randn(4, 16, device="cuda", requires_grad=True)
    saved = (a * out).sum()
    unpack_rows(table, fmt, out=out)
    with pytest.raises(RuntimeError, match=CHANGED):
        saved.backward()


def test_an_output_that_requires_a_gradient_is_refused():
    fmt = RowFormat(16, 8)
    table = pack_rows(torch.randn(4, 16, device="cuda"), fmt)
    out = torch.zeros(4, 16, device="cuda", requires_grad=True)
    for o in (out, out * 2):
        with pytest.raises(ValueError, match="grad"):
            unpack_rows(table, fmt, out=o)
    with torch.no_grad():
        assert torch.equal(unpack_rows(table, fmt, out=out), unpack_rows(table, fmt))


def test_in_inference_mode():
    """Tensors made there have no versions to count."""
    with torch.inference_mode():
        p = torch.randn(300, device="cuda")
        before = p.clone()
        AdamW([p]).step([torch.ones(300, device="cuda")])
        assert not torch.equal(p, before)
        fmt = RowFormat(16, 8)
        table = pack_rows(torch.randn(4, 16, device="cuda"), fmt)
        pack_rows(torch.randn(4, 16, device="cuda"), fmt, out=table)
        unpack_rows(table, fmt, out=torch.zeros(4, 16, device="cuda"))
