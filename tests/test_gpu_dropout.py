"""GPU: cdma_dropout / cdma_dropout_backward against the numpy oracle in 64 bits.

Which elements are dropped is exact.  The value x * scale + residual has three roundings in 32 bits (scale, product,
sum) and one to the type, so it may be off by 2^-22 (|x scale| + |residual|) + 2^-p |y|, p the type's bits."""
import numpy as np
import pytest
import torch

from oracle import dropout_numpy as dn
from oracle import gated_ffn as gf
from paper_1705_01626_b200 import binding as B
from tests.gpu_helpers import DT

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def normal(rows, cols, dtype, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, cols + pad, generator=g, device="cuda").to(dtype)[:, :cols]


def check(y, x, p, seed, sequence, residual=None):
    want = dn.dropout(x.double().cpu().numpy(), p, seed, sequence,
                      residual.double().cpu().numpy() if residual is not None else None)
    parts = np.abs(x.double().cpu().numpy()) * dn.scale(p)
    if residual is not None:
        parts = parts + np.abs(residual.double().cpu().numpy())
    got = y.double().cpu().numpy()
    bound = 2.0 ** -22 * parts + gf.UNIT[x.dtype] * np.abs(want) + gf.TINY[x.dtype]
    keep = dn.keep_mask(x.shape[0], x.shape[1], p, seed, sequence)
    there = np.zeros_like(got) if residual is None else residual.double().cpu().numpy()
    assert np.array_equal(got[~keep], there[~keep])
    assert (np.abs(got - want) <= bound).all()


def run(x, p, seed, sequence, residual=None, y=None, stream=0):
    rows, cols = x.shape
    if y is None:
        y = torch.full((rows, cols), 7.0, dtype=x.dtype, device="cuda")
    st = B.cdma_dropout(x.data_ptr(), x.stride(0), residual.data_ptr() if residual is not None else 0,
                        residual.stride(0) if residual is not None else 0, rows, cols, DT[x.dtype], p, seed, sequence,
                        y.data_ptr(), y.stride(0), stream)
    assert st == B.OK, B.status_string(st)
    torch.cuda.synchronize()
    return y


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (1, 8), (1, 9), (3, 5), (2, 64), (5, 1000), (7, 1001), (129, 24),
                                       (1, 100_003), (1000, 1), (33, 2055)])
def test_matches_the_oracle(dtype, rows, cols):
    x, r = normal(rows, cols, dtype, rows + cols), normal(rows, cols, dtype, rows + cols + 1)
    for p, seed, seq in [(0.1, 3, 4), (0.5, (1 << 63) + 12345, (1 << 40) + 7)]:
        check(run(x, p, seed, seq), x, p, seed, seq)
        check(run(x, p, seed, seq, r), x, p, seed, seq, r)
        dx = torch.full_like(x, 7.0)
        assert B.cdma_dropout_backward(x.data_ptr(), x.stride(0), rows, cols, DT[dtype], p, seed, seq, dx.data_ptr(),
                                       dx.stride(0), 0) == B.OK
        torch.cuda.synchronize()
        check(dx, x, p, seed, seq)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols,pads", [(64, (8, 16, 24)), (64, (1, 2, 3)), (61, (3, 11, 0)), (1001, (0, 7, 1))])
def test_row_strides_and_untouched_padding(dtype, cols, pads):
    rows = 37
    x, r = normal(rows, cols, dtype, 1, pads[0]), normal(rows, cols, dtype, 2, pads[1])
    wide = torch.full((rows, cols + pads[2]), 7.0, dtype=dtype, device="cuda")
    check(run(x, 0.25, 8, 9, r, wide[:, :cols]), x, 0.25, 8, 9, r)
    assert (wide[:, cols:] == 7.0).all()


def test_extreme_rates():
    x = normal(5, 333, torch.float32, 4)
    assert torch.equal(run(x, 0.0, 1, 2), x)
    x[0, 0], x[1, 5] = float("nan"), float("inf")
    assert (run(x, 1.0, 1, 2) == 0).all()
    tiny = 0.4 / 65536                    # rounds to no drops at all
    assert torch.equal(run(x[4:], tiny, 1, 2), x[4:])        # row 4 starts on 16 bytes


@pytest.mark.parametrize("cols", [512, 509])
def test_dropped_elements_are_zero_whatever_they_hold(cols):
    keep = torch.from_numpy(dn.keep_mask(16, cols, 0.5, 5, 6)).cuda()
    for value in (float("nan"), float("inf"), -float("inf"), -0.0):
        for dtype in DTYPES:
            x = torch.where(keep, 1.0, value).to(dtype)
            y = run(x, 0.5, 5, 6)
            assert torch.equal(y, keep.to(dtype) * 2)
            assert not torch.signbit(y).any()
    x = torch.full((16, cols), float("nan"), device="cuda")
    assert torch.equal(torch.isnan(run(x, 0.5, 5, 6)), keep)


@pytest.mark.parametrize("cols", [256, 255])
def test_in_place_and_on_another_stream(cols):
    x, r = normal(70, cols, torch.bfloat16, 5), normal(70, cols, torch.bfloat16, 6)
    stream = torch.cuda.Stream()
    want = run(x, 0.3, 1, 2, r, stream=stream.cuda_stream)
    a, b = x.clone(), r.clone()
    assert torch.equal(run(a, 0.3, 1, 2, r, y=a), want)
    assert torch.equal(run(x, 0.3, 1, 2, b, y=b), want)


def test_past_thirty_two_bits():
    # one row, and many rows, of more than 2^32 elements: the last ones against the oracle
    n = (1 << 32) + 1008
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    assert B.cdma_dropout(x.data_ptr(), 0, 0, 0, 1, n, B.BF16, 0.5, 11, 12, x.data_ptr(), 0, 0) == B.OK
    tail = (x[-2000:].float() / 2).cpu().numpy()
    assert np.array_equal(tail, dn.keep_mask(1, 2000, 0.5, 11, 12, first_block=(n - 2000) // 8)[0])
    x.fill_(1.0)
    rows = n // 16
    assert B.cdma_dropout(x.data_ptr(), 0, 0, 0, rows, 16, B.BF16, 0.5, 11, 12, x.data_ptr(), 0, 0) == B.OK
    tail = (x[rows * 16 - 1600: rows * 16].float() / 2).cpu().numpy().reshape(100, 16)
    assert np.array_equal(tail, dn.keep_mask(100, 16, 0.5, 11, 12, first_row=rows - 100))
    for cols in (1001, 9):                # rows that do not start on 16 bytes, long and short ones
        x.fill_(1.0)
        rows = n // cols
        assert B.cdma_dropout(x.data_ptr(), 0, 0, 0, rows, cols, B.BF16, 0.5, 11, 12, x.data_ptr(), 0, 0) == B.OK
        tail = (x[(rows - 100) * cols: rows * cols].float() / 2).cpu().numpy().reshape(100, cols)
        assert np.array_equal(tail, dn.keep_mask(100, cols, 0.5, 11, 12, first_row=rows - 100))
        assert (x[rows * cols:] == 1.0).all()


def test_dropped_maps_go_through_the_codec():
    x = normal(64, 1000, torch.float16, 9).relu()
    y = run(x, 0.5, 3, 3)
    n = y.numel()
    cap, ws_bytes = B.cdma_zvc_max_compressed_bytes(n, B.F16), B.cdma_zvc_workspace_bytes(n, B.F16)
    payload = torch.empty(cap, dtype=torch.uint8, device="cuda")
    table = torch.empty(B.cdma_zvc_table_entries(n), dtype=torch.int64, device="cuda")
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    c = B.cdma_zvc_compress(y.data_ptr(), n, B.F16, B.NCHW, payload.data_ptr(), cap, table.data_ptr(), ws.data_ptr(), ws_bytes, 0)
    assert c == 4 * (n // 32) + 2 * int((y != 0).sum())
