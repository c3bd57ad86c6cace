"""CPU: what the operators' entry points refuse, and their workspace sizes.  No kernel is launched: every call here
fails its checks (host memory stands in for device memory)."""
import ctypes

import pytest

from paper_1705_01626_b200 import binding as B


def host_buffer(size):
    buf = (ctypes.c_uint8 * (size + 256))()
    return buf, (ctypes.addressof(buf) + 255) // 256 * 256


def test_dropout_refusals():
    keep, base = host_buffer(8192)
    args = dict(d_x=base, ld_x=16, d_residual=0, ld_residual=0, rows=4, cols=16, dtype=B.F32, p=0.5, seed=1, sequence=2,
                d_y=base + 4096, ld_y=16)
    for change, want in [
        (dict(dtype=B.U8), B.ERR_UNSUPPORTED_DTYPE), (dict(dtype=9), B.ERR_UNSUPPORTED_DTYPE),
        (dict(p=-0.1), B.ERR_INVALID_ARG), (dict(p=1.01), B.ERR_INVALID_ARG), (dict(p=float("nan")), B.ERR_INVALID_ARG),
        (dict(d_x=0), B.ERR_INVALID_ARG), (dict(d_y=0), B.ERR_INVALID_ARG), (dict(ld_x=15), B.ERR_INVALID_ARG),
        (dict(ld_y=3), B.ERR_INVALID_ARG), (dict(d_residual=base + 1024, ld_residual=8), B.ERR_INVALID_ARG),
        (dict(d_x=base + 4), B.ERR_ALIGNMENT), (dict(d_y=base + 4098), B.ERR_ALIGNMENT),
        (dict(d_residual=base + 1028), B.ERR_ALIGNMENT),
        (dict(d_y=base + 16), B.ERR_INVALID_ARG),                    # overlaps x without being x
        (dict(d_y=base, ld_y=32), B.ERR_INVALID_ARG),                # x itself, but with another stride
        (dict(d_residual=base + 4096 + 32), B.ERR_INVALID_ARG),
        (dict(rows=1 << 32), B.ERR_INVALID_ARG), (dict(cols=1 << 35, ld_x=0, ld_y=0), B.ERR_INVALID_ARG),
        (dict(rows=1 << 30, cols=1 << 20, ld_x=0, ld_y=0), B.ERR_INVALID_ARG),
    ]:
        assert B.cdma_dropout(**{**args, **change}) == want, change
    assert B.cdma_dropout_backward(base, 15, 4, 16, B.F32, 0.5, 1, 2, base + 4096, 16) == B.ERR_INVALID_ARG
    assert B.cdma_dropout(**{**args, "rows": 0, "d_x": 0, "d_y": 0}) == B.OK        # nothing to do
    assert B.cdma_dropout(**{**args, "cols": 0, "d_x": 0, "d_y": 0, "ld_x": 0, "ld_y": 0}) == B.OK


def desc(**change):
    return B.cdma_gated_ffn_desc(**{**dict(m=4, k=8, f=16, dtype=B.BF16, activation=B.ACT_SILU), **change})


def test_gated_ffn_refusals():
    keep, base = host_buffer(1 << 16)
    x, wg, wu, h, ws = base, base + 1024, base + 2048, base + 4096, base + 8192
    dh, dx, dwg, dwu = base + 5120, base + 6144, base + 6656, base + 7168
    size = 32768
    result = (ctypes.c_uint64 * 2)()

    def fwd(d=None, x=x, wg=wg, wu=wu, h=h, ws=ws, size=size):
        return B.cdma_gated_ffn_forward(d if d is not None else desc(), x, wg, wu, h, ws, size)

    def bwd(d=None, x=x, wg=wg, wu=wu, dh=dh, dx=dx, dwg=dwg, dwu=dwu, ws=ws, size=size):
        return B.cdma_gated_ffn_backward(d if d is not None else desc(), x, wg, wu, dh, dx, dwg, dwu, ws, size)

    for change, want in [
        (dict(dtype=B.U8), B.ERR_UNSUPPORTED_DTYPE), (dict(dtype=-1), B.ERR_UNSUPPORTED_DTYPE),
        (dict(activation=3), B.ERR_INVALID_ARG), (dict(dropout_p=1.5), B.ERR_INVALID_ARG),
        (dict(dropout_p=float("nan")), B.ERR_INVALID_ARG), (dict(m=1 << 31), B.ERR_INVALID_ARG),
        (dict(k=(1 << 21) + 1), B.ERR_INVALID_ARG), (dict(f=(1 << 21) + 1), B.ERR_INVALID_ARG),
        (dict(ld_x=7), B.ERR_INVALID_ARG), (dict(ld_wg=7), B.ERR_INVALID_ARG), (dict(ld_wu=7), B.ERR_INVALID_ARG),
        (dict(ld_h=15), B.ERR_INVALID_ARG), (dict(ld_dx=7), B.ERR_INVALID_ARG), (dict(ld_dw=7), B.ERR_INVALID_ARG),
        (dict(ld_x=(1 << 31) + 1), B.ERR_INVALID_ARG),
    ]:
        assert fwd(desc(**change)) == -want and bwd(desc(**change)) == -want, change
        assert B.cdma_gated_ffn_workspace_bytes(desc(**change), 0) == 0
    assert B.cdma_gated_ffn_forward(None, x, wg, wu, h, ws, size) == -B.ERR_INVALID_ARG
    assert B.cdma_gated_ffn_workspace_bytes(None, 1) == 0
    for name in ("x", "wg", "wu", "h", "ws"):
        assert fwd(**{name: 0}) == -B.ERR_INVALID_ARG, name
        assert fwd(**{name: {"x": x, "wg": wg, "wu": wu, "h": h, "ws": ws}[name] + 8}) == -B.ERR_ALIGNMENT, name
    for name in ("x", "wg", "wu", "dh", "dwg", "dwu", "ws"):
        assert bwd(**{name: 0}) == -B.ERR_INVALID_ARG, name
    assert bwd(dx=0, dwg=0, dwu=0) == -B.ERR_INVALID_ARG
    assert bwd(dx=dx + 2) == -B.ERR_ALIGNMENT
    assert fwd(size=8) == -B.ERR_BUFFER_TOO_SMALL
    assert bwd(size=B.cdma_gated_ffn_workspace_bytes(desc(), 1) - 1) == -B.ERR_BUFFER_TOO_SMALL
    for name in ("x", "wg", "wu", "ws"):            # the output over an input or the workspace
        at = {"x": x, "wg": wg, "wu": wu, "ws": ws}[name]
        assert fwd(h=at) == -B.ERR_INVALID_ARG, name
        assert bwd(dx=at) == -B.ERR_INVALID_ARG and bwd(dwg=at) == -B.ERR_INVALID_ARG, name
    assert bwd(dwu=dwg) == -B.ERR_INVALID_ARG and bwd(dx=dh) == -B.ERR_INVALID_ARG
    assert fwd(x=ws + 256) == -B.ERR_INVALID_ARG
    st = B.cdma_gated_ffn_forward_async(desc(), x, wg, wu, h, ws, size, 0, 0)
    assert st == B.ERR_INVALID_ARG                  # no place for the result words
    del result


def test_gated_ffn_workspace():
    for dtype, s in ((B.F32, 4), (B.F16, 2), (B.BF16, 2)):
        for m, k, f in ((1, 8, 16), (300, 1001, 77), (8192, 4096, 10944)):
            d = desc(m=m, k=k, f=f, dtype=dtype)
            fwd, bwd = B.cdma_gated_ffn_workspace_bytes(d, 0), B.cdma_gated_ffn_workspace_bytes(d, 1)
            assert fwd >= 256 and fwd % 256 == 0 and bwd % 256 == 0
            assert bwd >= 2 * m * f * s             # the gradients of G and U


def test_gated_ffn_workspace_of_empty_blocks():
    for m, k, f in ((0, 8, 16), (4, 0, 16), (4, 8, 0), (0, 0, 0)):
        for dtype in (B.F32, B.F16):
            for backward in (0, 1):
                assert B.cdma_gated_ffn_workspace_bytes(desc(m=m, k=k, f=f, dtype=dtype), backward) >= 256
