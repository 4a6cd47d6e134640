"""Rows held in 8 and 4 bits (pack_rows, unpack_rows): codes and floats against
the formula's fp32 steps, bit for bit, and what they stand for against the
source in 64 bits."""
import numpy as np
import pytest
import torch

import plain_operators as plain
from paper_2410_22697_amd import RowFormat, pack_rows, unpack_rows

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows_of(n, d, seed, kind="normal"):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, d)) * np.exp(rng.uniform(-6, 6, (n, 1)))
    if kind == "relu":
        x = np.maximum(x, 0)
    return x.astype(np.float32)


def expected_bytes(x, fmt):
    codes, lo, step = plain.pack(x, fmt.bits, fmt.group)
    return plain.to_bytes(codes, lo, step, fmt.bits), plain.stand_for(codes, lo, step, fmt.group), step


def check(x32, fmt, table, slots=None):
    """The table's rows hold exactly the formula's codes and floats for x32."""
    want, values, step = expected_bytes(x32, fmt)
    got = table.cpu().numpy()
    got = got if slots is None else got[slots]
    assert np.array_equal(got[:len(want), :fmt.least_bytes], want)
    return values, step


@pytest.mark.parametrize("d", [1, 2, 3, 7, 8, 9, 31, 64, 100, 128, 257, 512, 513, 1000, 1537])
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("group", [0, 16, 64, 512])
def test_codes_floats_and_values(d, bits, group):
    for dtype in TYPES.values():
        x = torch.from_numpy(rows_of(37, d, d * 7 + bits, "relu" if group == 16 else "normal")).to(dtype).cuda()
        fmt = RowFormat(d, bits, group)
        table = pack_rows(x, fmt)
        x32 = x.float().cpu().numpy()
        values, step = check(x32, fmt, table)
        got = unpack_rows(table, fmt).cpu().numpy().astype(np.float64)
        # one product, or a product and a sum (fused or not), rounded to fp32
        assert np.all(np.abs(got - values) <= 2 * plain.EPS * (np.abs(values) + 2 * np.abs(x32).max(1, keepdims=True)))
        # the nearest code: half a step, and what the reciprocal's and the product's roundings shift a tie by
        widest = np.concatenate([np.repeat(step[:, g:g + 1], b - a, 1)
                                 for g, (a, b) in enumerate(plain.groups_of(d, group))], 1).astype(np.float64)
        assert np.all(np.abs(got - x32) <= widest * (0.5 + 1e-4) + 4 * plain.EPS * np.abs(x32).max(1, keepdims=True))
        half = unpack_rows(table, fmt, dtype=torch.bfloat16)
        assert torch.equal(half, unpack_rows(table, fmt).to(torch.bfloat16))


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n", [0, 1, 3, 1000])
def test_slots_and_index(bits, n):
    """Slots in any order, some outside the table (left out); an index outside reads zeros; other rows stay."""
    d, rows = 50, 700
    fmt = RowFormat(d, bits, 16)
    rng = np.random.default_rng(n)
    x = rows_of(n, d, n)
    slots = rng.permutation(2 * rows)[:n].astype(np.int32) - 100  # in the table, below it and behind it
    table = torch.full((rows, fmt.row_bytes), 7, dtype=torch.uint8, device="cuda")
    pack_rows(torch.from_numpy(x).cuda(), fmt, out=table, slots=torch.from_numpy(slots).cuda())
    got = table.cpu().numpy()
    inside = (slots >= 0) & (slots < rows)
    want, values, _ = expected_bytes(x, fmt)
    assert np.array_equal(got[slots[inside]], want[inside])
    untouched = np.setdiff1d(np.arange(rows), slots[inside])
    assert np.all(got[untouched] == 7)
    if not n:
        assert unpack_rows(table, fmt, index=torch.zeros(0, dtype=torch.int32, device="cuda")).shape == (0, d)
        return
    read = unpack_rows(table, fmt, index=torch.from_numpy(slots).cuda()).cpu().numpy()
    assert np.all(read[~inside] == 0)
    assert np.allclose(read[inside], values[inside], rtol=1e-6, atol=1e-6 * np.abs(x).max())
    # the least and the largest index there is
    ends = torch.tensor([-2 ** 31, 2 ** 31 - 1, -1, rows], dtype=torch.int32, device="cuda")
    assert torch.all(unpack_rows(table, fmt, index=ends) == 0)


@pytest.mark.parametrize("bits", [8, 4])
def test_special_values(bits):
    d = 40
    base = rows_of(12, d, 5)
    x = base.copy()
    x[0] = 0
    x[1] = -3.25                       # a constant: 4 bits hold it exactly
    x[2] *= 2.0 ** -140                # under every code's reach
    x[3, 3] = np.inf
    x[4, 20] = -np.inf
    x[5, 39] = np.nan
    x[6, :2] = [3.3e38, -3.3e38]       # finite, their difference is not
    x[7] = np.where(np.arange(d) % 2, -0.0, 0.0)
    x[8] = 2.0 ** -119
    x[9, 0] = 1e30                     # one value so large that all others round to code 0 (8 bits)
    fmt = RowFormat(d, bits, 16)
    table = pack_rows(torch.from_numpy(x).cuda(), fmt)
    want, values, _ = expected_bytes(x, fmt)
    got, floats = table.cpu().numpy(), fmt.floats_at
    assert np.array_equal(got[:, :floats], want[:, :floats])
    a, b = got[:, floats:].copy().view(np.float32), want[:, floats:].copy().view(np.float32)
    assert np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(a[~np.isnan(a)], b[~np.isnan(b)])
    read = unpack_rows(table, fmt).cpu().numpy()
    assert np.array_equal(np.isnan(read), np.isnan(values))
    assert np.isnan(read[3, :16]).all() and np.isfinite(read[3, 16:]).all()  # its group only
    if bits == 4:
        assert np.all(read[1] == -3.25) and np.isnan(read[6, :16]).all()
    else:
        assert np.isfinite(read[6]).all()


def test_padded_rows_strided_sources_and_outputs():
    d = 60
    for bits in (8, 4):
        fmt = RowFormat(d, bits, 0, row_bytes=128)
        wide = torch.from_numpy(rows_of(33, 2 * d + 3, 1)).cuda()
        x = wide[:, 3:3 + d]  # rows at odd offsets, of an odd stride
        table = torch.full((33, 128), 9, dtype=torch.uint8, device="cuda")
        pack_rows(x, fmt, out=table)
        values, _ = check(x.cpu().numpy(), fmt, table)
        assert torch.all(table[:, fmt.least_bytes:] == 9)  # padding is not written
        out = torch.full((33, d + 5), 4.0, device="cuda")
        unpack_rows(table, fmt, out=out[:, 1:1 + d])
        assert torch.equal(out[:, 1:1 + d], unpack_rows(table, fmt))
        assert torch.all(out[:, 0] == 4) and torch.all(out[:, 1 + d:] == 4)
        half = wide.bfloat16()[:, 1:1 + d]
        check(half.float().cpu().numpy(), fmt, pack_rows(half, fmt))


def test_table_beyond_32_bits():
    fmt = RowFormat(256, 8)
    rows = (1 << 32) // fmt.row_bytes + 1000
    table = torch.empty((rows, fmt.row_bytes), dtype=torch.uint8, device="cuda")
    x = rows_of(64, 256, 3)
    slots = torch.arange(rows - 64, rows, dtype=torch.int32, device="cuda")
    pack_rows(torch.from_numpy(x).cuda(), fmt, out=table, slots=slots)
    check(x, fmt, table[-64:])
    assert torch.equal(unpack_rows(table, fmt, index=slots), unpack_rows(table[-64:].clone(), fmt))


def test_pinned_table_is_read_in_place():
    fmt = RowFormat(100, 8)
    table = pack_rows(torch.from_numpy(rows_of(500, 100, 4)).cuda(), fmt)
    pinned = torch.empty(table.shape, dtype=torch.uint8, pin_memory=True)
    pinned.copy_(table)
    index = torch.randint(0, 500, (300,), dtype=torch.int32, device="cuda")
    assert torch.equal(unpack_rows(pinned, fmt, index=index), unpack_rows(table, fmt, index=index))


def test_on_another_stream():
    fmt = RowFormat(128, 8)
    x = torch.randn(20000, 128, device="cuda")
    want = unpack_rows(pack_rows(x, fmt), fmt)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = unpack_rows(pack_rows(x, fmt), fmt)
    side.synchronize()
    assert torch.equal(got, want)


def test_refusals():
    fmt = RowFormat(16, 8)
    x = torch.zeros(4, 16, device="cuda")
    table = torch.zeros(4, fmt.row_bytes, dtype=torch.uint8, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (lambda: pack_rows(x.half(), fmt), lambda: pack_rows(x[:, :8], fmt), lambda: pack_rows(x.t(), fmt),
                lambda: pack_rows(x, fmt, out=table[:, :8]), lambda: pack_rows(x, fmt, out=table[:2]),
                lambda: pack_rows(x, fmt, out=table, slots=ids.long()), lambda: pack_rows(x, fmt, out=table, slots=ids[:3]),
                lambda: pack_rows(x, fmt, slots=ids), lambda: pack_rows(x[:1].expand(4, 16), fmt), lambda: pack_rows(x.cpu(), fmt),
                lambda: unpack_rows(table.cpu(), fmt), lambda: unpack_rows(table, fmt, index=ids[::2]),
                lambda: unpack_rows(table, fmt, dtype=torch.float16), lambda: unpack_rows(table, fmt, out=x[:3]),
                lambda: unpack_rows(table, fmt, out=x[:1].expand(4, 16))):
        with pytest.raises(ValueError):
            bad()
