"""GPU: cdma_gated_ffn_forward / _backward against the formulas in 64 bits, element by element within the bounds that
oracle/gated_ffn.py derives; the padding of every strided output and the bytes behind the workspace stay untouched."""
import math

import pytest
import torch

from oracle import dropout_numpy as dn
from oracle import gated_ffn as gf
from paper_1705_01626_b200 import binding as B
from tests.gpu_helpers import CANARY, DT

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
ACTS = {"relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}


class Block:
    """Inputs and outputs of one call; pads: extra columns of x, Wg, Wu, h/dh, dx, dWg/dWu."""

    def __init__(self, m, k, f, dtype, act="silu", p=0.0, seed=5, sequence=6, pads=(0, 0, 0, 0, 0, 0), rng=1):
        self.m, self.k, self.f, self.dtype, self.act, self.p, self.seed, self.sequence = m, k, f, dtype, act, p, seed, sequence
        g = torch.Generator(device="cuda").manual_seed(rng + 7 * m + 11 * k + 13 * f)

        def wide(rows, cols, pad, scale=None):
            t = torch.full((rows, cols + pad), 7.0, dtype=dtype, device="cuda")
            if scale is not None:
                t[:, :cols] = (torch.randn(rows, cols, generator=g, device="cuda") * scale).to(dtype)
            return t

        self.xw, self.wgw, self.wuw = wide(m, k, pads[0], 1.0), wide(f, k, pads[1], max(k, 1) ** -0.5), wide(f, k, pads[2], max(k, 1) ** -0.5)
        self.dhw = wide(m, f, pads[3], 0.1)
        self.hw, self.dxw = wide(m, f, pads[3]), wide(m, k, pads[4])
        self.dwgw, self.dwuw = wide(f, k, pads[5]), wide(f, k, pads[5])
        self.x, self.wg, self.wu, self.dh = self.xw[:, :k], self.wgw[:, :k], self.wuw[:, :k], self.dhw[:, :f]
        self.desc = B.cdma_gated_ffn_desc(
            m=m, k=k, f=f, ld_x=k + pads[0], ld_wg=k + pads[1], ld_wu=k + pads[2], ld_h=f + pads[3], ld_dx=k + pads[4],
            ld_dw=k + pads[5], dtype=DT[dtype], activation=ACTS[act], dropout_p=p, dropout_seed=seed, dropout_sequence=sequence)

    ws_shift = 0        # bytes of the workspace's start past 512

    def workspace(self, backward):
        self.ws_bytes = B.cdma_gated_ffn_workspace_bytes(self.desc, backward)
        self.ws = torch.full((self.ws_shift + self.ws_bytes + 256,), CANARY, dtype=torch.uint8, device="cuda")[self.ws_shift:]

    def forward(self, stream=0):
        self.workspace(0)
        r = B.cdma_gated_ffn_forward(self.desc, self.x.data_ptr(), self.wg.data_ptr(), self.wu.data_ptr(), self.hw.data_ptr(),
                                     self.ws.data_ptr(), self.ws_bytes, stream)
        assert r == self.m * self.f * self.x.element_size(), B.status_string(r)
        assert (self.ws[self.ws_bytes:] == CANARY).all() and (self.hw[:, self.f:] == 7.0).all()
        return self.hw[:, :self.f]

    def backward(self, stream=0, dx=True, dw=True):
        self.workspace(1)
        r = B.cdma_gated_ffn_backward(self.desc, self.x.data_ptr(), self.wg.data_ptr(), self.wu.data_ptr(), self.dh.data_ptr(),
                                      self.dxw.data_ptr() if dx else 0, self.dwgw.data_ptr() if dw else 0,
                                      self.dwuw.data_ptr() if dw else 0, self.ws.data_ptr(), self.ws_bytes, stream)
        assert r == self.x.element_size() * ((self.m * self.k if dx else 0) + (2 * self.f * self.k if dw else 0)), B.status_string(r)
        assert (self.ws[self.ws_bytes:] == CANARY).all()
        for t in (self.dxw, self.dwgw, self.dwuw):
            assert (t[:, self.k:] == 7.0).all()
        return {"dx": self.dxw[:, :self.k], "dwg": self.dwgw[:, :self.k], "dwu": self.dwuw[:, :self.k]}

    def check_forward(self, stream=0):
        h = self.forward(stream)
        want = gf.forward(self.x, self.wg, self.wu, self.act, self.p, self.seed, self.sequence)
        within(h, want, "h")
        return h

    def check_backward(self, stream=0):
        got = self.backward(stream)
        want = gf.backward(self.x, self.wg, self.wu, self.dh, self.act, self.p, self.seed, self.sequence)
        for n in got:
            within(got[n], want, n)
        return got


def within(got, want, name):
    off = (got.double() - want.value[name]).abs()
    worst = (off / want.bound[name].clamp(min=1e-300)).max() if off.numel() else 0
    assert torch.isfinite(got).all() and worst <= 1, "%s: %.3g of its bound" % (name, float(worst))


SIZES = [(1, 1, 1), (1, 64, 128), (1, 1000, 77), (2, 33, 5), (3, 64, 256), (7, 200, 130), (16, 512, 256), (17, 1024, 136),
         (31, 72, 1000), (33, 128, 64), (64, 256, 512), (65, 136, 129), (127, 65, 127), (128, 64, 128), (129, 130, 131),
         (200, 512, 384), (255, 257, 259), (256, 128, 256), (257, 192, 520), (300, 1001, 311), (513, 320, 640)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,k,f", SIZES)
def test_matches_the_formulas(m, k, f, dtype):
    act = ("relu", "silu", "gelu")[(m + k + f) % 3]
    p = (0.0, 0.25)[(m + f) % 2]
    b = Block(m, k, f, dtype, act, p)
    b.check_forward()
    b.check_backward()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("m", [1, 5, 40, 300])
def test_activations_and_dropout(act, dtype, m):
    for p in (0.0, 0.5):
        b = Block(m, 128, 264, dtype, act, p, seed=(1 << 60) + m, sequence=(7 << 35) + 1)
        b.check_forward()
        b.check_backward()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 20, 150])
@pytest.mark.parametrize("pads", [(8, 16, 24, 32, 40, 48), (1, 2, 3, 4, 5, 6), (4, 4, 4, 4, 4, 4), (0, 3, 0, 1, 0, 0)])
def test_strides(dtype, m, pads):
    for k, f in ((128, 256), (67, 141)):
        b = Block(m, k, f, dtype, "gelu", 0.1, pads=pads)
        b.check_forward()
        b.check_backward()


@pytest.mark.parametrize("dtype", DTYPES)
def test_both_projections_in_one_weight_buffer(dtype):
    # gate and up projections as the halves of one [f, 2k] buffer, by rows of it, and their gradients likewise
    m, k, f = 70, 64, 96
    b = Block(m, k, f, dtype, "silu")
    both = torch.cat((b.wg, b.wu), dim=1).contiguous()
    grads = torch.zeros_like(both)
    desc = B.cdma_gated_ffn_desc(m=m, k=k, f=f, ld_wg=2 * k, ld_wu=2 * k, ld_dw=2 * k, dtype=DT[dtype], activation=B.ACT_SILU)
    ws = torch.empty(B.cdma_gated_ffn_workspace_bytes(desc, 1), dtype=torch.uint8, device="cuda")
    r = B.cdma_gated_ffn_backward(desc, b.x.data_ptr(), both.data_ptr(), both[:, k:].data_ptr(), b.dh.data_ptr(), b.dxw.data_ptr(),
                                  grads.data_ptr(), grads[:, k:].data_ptr(), ws.data_ptr(), ws.numel(), 0)
    assert r > 0, B.status_string(r)
    want = gf.backward(b.x, b.wg, b.wu, b.dh, "silu")
    for got, n in ((b.dxw, "dx"), (grads[:, :k], "dwg"), (grads[:, k:], "dwu")):
        within(got, want, n)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 40, 300])
def test_closed_gates_and_dropped_places_are_positive_zeros(dtype, m):
    # the codec compresses bit patterns: -0 would be kept
    h = Block(m, 96, 264, dtype, "relu", 0.25).forward()
    zero = h == 0
    assert 0.5 < zero.double().mean() < 0.8
    assert not torch.signbit(h[zero]).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [3, 90])
def test_dropout_is_that_of_the_dropout_call(dtype, m):
    k, f, p = 96, 203, 0.4
    plain, dropped = Block(m, k, f, dtype, "relu"), Block(m, k, f, dtype, "relu", p)
    h = plain.forward()
    y = torch.empty_like(h, memory_format=torch.contiguous_format)
    assert B.cdma_dropout(h.data_ptr(), h.stride(0), 0, 0, m, f, DT[dtype], p, 5, 6, y.data_ptr(), f, 0) == B.OK
    got = dropped.forward()
    assert torch.equal(got == 0, y == 0)
    # h rounded before and after the factor instead of after it alone
    assert ((got.double() - y.double()).abs() <= 3 * gf.UNIT[dtype] * y.double().abs() + 2 * gf.TINY[dtype]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [2, 140])
def test_parts_of_the_gradient(dtype, m):
    b = Block(m, 80, 120, dtype)
    both = {n: t.clone() for n, t in b.backward().items()}
    b.dxw.fill_(7.0)
    b.dwgw.fill_(7.0)
    b.dwuw.fill_(7.0)
    assert torch.equal(b.backward(dw=False)["dx"], both["dx"]) and (b.dwgw == 7.0).all() and (b.dwuw == 7.0).all()
    b.dxw.fill_(7.0)
    got = b.backward(dx=False)
    assert torch.equal(got["dwg"], both["dwg"]) and torch.equal(got["dwu"], both["dwu"]) and (b.dxw == 7.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift", [16, 240])
def test_workspaces_anywhere_on_sixteen_bytes(dtype, shift):
    for m in (20, 150, 300):            # split products with sums in the workspace among them
        b = Block(m, 1001, 520, dtype, "silu")
        b.ws_shift = shift
        b.check_forward()
        b.check_backward()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 20, 300])
def test_calls_in_a_graph(dtype, m):
    b = Block(m, 264, 520, dtype, "relu", 0.25)
    want, grads = b.forward().clone(), {n: t.clone() for n, t in b.backward().items()}
    words = torch.zeros(2, dtype=torch.int64).pin_memory()
    y = torch.empty(m, 520, dtype=dtype, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        assert B.cdma_gated_ffn_forward_async(b.desc, b.x.data_ptr(), b.wg.data_ptr(), b.wu.data_ptr(), b.hw.data_ptr(),
                                              b.ws.data_ptr(), b.ws_bytes, s, words.data_ptr()) == B.OK
        assert B.cdma_dropout(b.hw.data_ptr(), 520, 0, 0, m, 520, DT[dtype], 0.0, 1, 2, y.data_ptr(), 520, s) == B.OK
        assert B.cdma_gated_ffn_backward_async(b.desc, b.x.data_ptr(), b.wg.data_ptr(), b.wu.data_ptr(), b.dh.data_ptr(),
                                               b.dxw.data_ptr(), b.dwgw.data_ptr(), b.dwuw.data_ptr(), b.ws.data_ptr(),
                                               b.ws_bytes, s, words.data_ptr()) == B.OK
    for _ in range(3):
        for t in (b.hw, y, b.dxw, b.dwgw, b.dwuw):
            t.fill_(7.0)
        words.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.hw, want) and torch.equal(y, want)
        assert torch.equal(b.dxw, grads["dx"]) and torch.equal(b.dwgw, grads["dwg"]) and torch.equal(b.dwuw, grads["dwu"])
        assert int(words[1]) == 0 and int(words[0]) > 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_inputs_written_right_before_the_call(dtype):
    # launches begin before the kernel in front has ended: what that kernel writes has to be what is read
    for m in (1, 2, 20, 300):
        b = Block(m, 512, 1024, dtype, "silu")
        b.workspace(0)
        stream = torch.cuda.current_stream().cuda_stream
        words = torch.zeros(2, dtype=torch.int64).pin_memory()
        x, outs = b.x.clone(), []
        for i in range(20):
            b.x.copy_(x)
            b.x.mul_(1.0 + i)
            assert B.cdma_gated_ffn_forward_async(b.desc, b.x.data_ptr(), b.wg.data_ptr(), b.wu.data_ptr(), b.hw.data_ptr(),
                                                  b.ws.data_ptr(), b.ws_bytes, stream, words.data_ptr()) == B.OK
            outs.append(b.hw.clone())
        for i in (0, 7, 19):
            b.x.copy_(x)
            b.x.mul_(1.0 + i)
            torch.cuda.synchronize()
            assert torch.equal(b.forward(), outs[i])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,k,f", [(40, 512, 640), (130, 257, 391), (513, 320, 640)])
def test_nothing_is_read_before_it_is_written(m, k, f, dtype):
    # the workspace holds NaNs in front of every call: a gradient that one kernel reads before another wrote it would show
    b = Block(m, k, f, dtype, "relu", 0.25)
    want = {n: t.clone() for n, t in b.backward().items()}
    stream = torch.cuda.current_stream().cuda_stream
    words = torch.zeros(2, dtype=torch.int64).pin_memory()
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    flush = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    for i in range(400):
        if i % 4 == 0:
            flush.fill_(i & 127)
        b.ws[:b.ws_bytes].fill_(0x7f if dtype == torch.float16 else 0xff)
        assert B.cdma_gated_ffn_backward_async(b.desc, b.x.data_ptr(), b.wg.data_ptr(), b.wu.data_ptr(), b.dh.data_ptr(),
                                               b.dxw.data_ptr(), b.dwgw.data_ptr(), b.dwuw.data_ptr(), b.ws.data_ptr(),
                                               b.ws_bytes, stream, words.data_ptr()) == B.OK
        for n, t in (("dx", b.dxw), ("dwg", b.dwgw), ("dwu", b.dwuw)):
            wrong += (t[:, :k] != want[n]).sum()
    assert int(wrong) == 0


@pytest.mark.parametrize("dtype", DTYPES)
def test_sizes_of_zero(dtype):
    for m, k, f in ((0, 8, 16), (4, 0, 16), (4, 8, 0), (0, 0, 0)):
        b = Block(m, k, f, dtype)
        assert (b.forward() == 0).all()
        for t in b.backward().values():
            assert (t == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [4, 300])
def test_same_bits_every_time_and_on_another_stream(dtype, m):
    b = Block(m, 300, 500, dtype, "gelu", 0.1)
    h, grads = b.forward().clone(), {n: t.clone() for n, t in b.backward().items()}
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    assert torch.equal(b.forward(stream.cuda_stream), h)
    got = b.backward(stream.cuda_stream)
    assert all(torch.equal(got[n], grads[n]) for n in grads)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [6, 200])
def test_what_is_not_finite_stays_in_its_row(dtype, m):
    b = Block(m, 64, 96, dtype, "relu")
    clean = b.forward().clone()
    b.x[3, 5] = float("inf")
    b.x[4, 0] = float("nan")
    h = b.forward()
    rest = [r for r in range(m) if r not in (3, 4)]
    assert torch.equal(h[rest], clean[rest])
    assert torch.isnan(h[4]).all()          # a ReLU keeps NaNs
    assert not torch.isfinite(h[3]).all()


@pytest.mark.parametrize("m", [3, 130])
def test_dropped_places_are_zero_where_the_product_is_not_finite(m):
    b = Block(m, 64, 96, torch.bfloat16, "silu", 0.5)
    b.x[1] = float("nan")
    keep = torch.from_numpy(dn.keep_mask(m, 96, 0.5, 5, 6)).cuda()
    h = b.forward()
    assert torch.equal(torch.isnan(h[1]), keep[1]) and (h[1][~keep[1]] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [8, 130])
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_saturated_gates(dtype, m, act):
    # gates far out on both sides: e^-g overflows or vanishes, the outputs must not
    k, f = 32, 64
    b = Block(m, k, f, dtype, act)
    b.x.zero_(), b.wg.zero_()
    b.x[:, 0], b.x[:, 1] = 30.0, 1.0
    b.wg[: f // 2, 0], b.wg[f // 2:, 0] = 4.0, -4.0       # G = 120 and -120
    b.check_forward()
    b.check_backward()


def test_gradient_against_differences_of_the_forward_pass():
    # both passes in 32 bits; L = sum(h dh) along random directions, steps of 2^-6 and 2^-7 combined so that the
    # third-order term cancels; what is left is fifth-order and the rounding of h, each h off by its bound
    m, k, f = 12, 40, 56
    b = Block(m, k, f, torch.float32, "silu", 0.2)
    grads = b.check_backward()
    bound = float((gf.forward(b.x, b.wg, b.wu, "silu", 0.2, 5, 6).bound["h"] * b.dh.double().abs()).sum())
    g = torch.Generator(device="cuda").manual_seed(4)
    for name, t in (("dx", b.x), ("dwg", b.wg), ("dwu", b.wu)):
        v = torch.randn(t.shape, generator=g, device="cuda")
        v /= v.norm()
        keep = t.clone()

        def loss(step):
            t.copy_((keep.double() + step * v.double()).float())
            value = float((b.forward().double() * b.dh.double()).sum())
            moved = t.double() - keep.double()
            t.copy_(keep)
            return value, moved

        def slope(step):
            (up, a), (down, c) = loss(step), loss(-step)
            return (up - down) / (2 * step), (a - c) / (2 * step)

        (fine, vf), (coarse, vc) = slope(2.0 ** -7), slope(2.0 ** -6)
        diff = (4 * fine - coarse) / 3
        direction = (4 * vf - vc) / 3        # the step that the rounded inputs really took
        want = float((grads[name].double() * direction).sum())
        rounding = (4 * bound * 2.0 ** 7 + bound * 2.0 ** 6) / 3
        size = float((b.dh.double().abs().sum()))
        assert abs(diff - want) <= rounding + 2.0 ** -24 * size, (name, diff, want, rounding)


def test_result_words_of_the_async_forms():
    b = Block(50, 64, 96, torch.bfloat16)
    for pinned in (True, False):
        words = torch.full((2,), -1, dtype=torch.int64)
        words = words.pin_memory() if pinned else words
        b.workspace(1)
        st = B.cdma_gated_ffn_forward_async(b.desc, b.x.data_ptr(), b.wg.data_ptr(), b.wu.data_ptr(), b.hw.data_ptr(),
                                            b.ws.data_ptr(), b.ws_bytes, 0, words.data_ptr())
        torch.cuda.synchronize()
        assert st == B.OK and words.tolist() == [50 * 96 * 2, 0]
        st = B.cdma_gated_ffn_backward_async(b.desc, b.x.data_ptr(), b.wg.data_ptr(), b.wu.data_ptr(), b.dh.data_ptr(),
                                             b.dxw.data_ptr(), b.dwgw.data_ptr(), b.dwuw.data_ptr(), b.ws.data_ptr(),
                                             b.ws_bytes, 0, words.data_ptr())
        torch.cuda.synchronize()
        assert st == B.OK and words.tolist() == [2 * (50 * 64 + 2 * 96 * 64), 0]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_error_as_a_whole_at_ordinary_sizes(dtype):
    # the 2-norm of the error: one rounding of h, two of the gradients, each below 2^-p of a value
    b = Block(600, 1024, 1408, dtype, "silu")
    rel = lambda got, want: float((got.double() - want).norm() / want.norm())
    assert rel(b.forward(), gf.forward(b.x, b.wg, b.wu, "silu").value["h"]) < gf.UNIT[dtype] + 2.0 ** -18
    got, want = b.backward(), gf.backward(b.x, b.wg, b.wu, b.dh, "silu").value
    for n in got:
        assert rel(got[n], want[n]) < math.sqrt(2) * gf.UNIT[dtype] + 2.0 ** -18


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m", [128, 512])
def test_signs_of_gates_near_zero(dtype, m):
    # The gradient of a ReLU passes where G > 0.  x ends in the unit matrix and Wg and Wu in zeros there, so that the last
    # columns of dWg are dG itself.  The products are of size 2^-6 and their partial sums mostly below 1: added to nearest
    # in 32 bits, 128 to a lane and then across lanes, they are off by sqrt(133) 2^-26 = 1.7e-7 or so; a sum cut off 256
    # times is off by more than 1e-6.  Farther from zero than 2^-21 = 4.8e-7 every sign has to be that of the sum in 64 bits.
    k, f = 4096, 8192
    b = Block(m, k + m, f, dtype, "relu")
    b.x[:, k:] = torch.eye(m, device="cuda")
    b.wg[:, k:], b.wu[:, k:] = 0, 0
    b.dh.fill_(1.0)
    g = b.x[:, :k].double() @ b.wg[:, :k].double().t()
    u = b.x[:, :k].double() @ b.wu[:, :k].double().t()
    dg = b.backward(dx=False)["dwg"][:, k:].t()
    sure = (g.abs() > 2.0 ** -21) & (u.abs() > 2.0 ** -10)
    assert sure.double().mean() > 0.99
    assert torch.equal((dg != 0)[sure], (g > 0)[sure])


def test_maps_past_thirty_two_bits():
    # h, dh, dG and dU of more than 2^32 elements: the last rows and the last hidden columns against the formulas
    m, k, f, dtype = 270_000, 64, 16_000, torch.bfloat16
    b = Block(m, k, f, dtype, "silu")
    b.forward()
    last = slice(m - 64, m)
    want = gf.forward(b.x[last], b.wg, b.wu, "silu")
    within(b.hw[last], want, "h")
    del b.hw
    b.workspace(1)
    r = B.cdma_gated_ffn_backward(b.desc, b.x.data_ptr(), b.wg.data_ptr(), b.wu.data_ptr(), b.dhw.data_ptr(), b.dxw.data_ptr(),
                                  b.dwgw.data_ptr(), b.dwuw.data_ptr(), b.ws.data_ptr(), b.ws_bytes, 0)
    assert r == 2 * (m * k + 2 * f * k), B.status_string(r)
    within(b.dxw[last], gf.backward(b.x[last], b.wg, b.wu, b.dhw[last], "silu"), "dx")
    of = slice(f - 32, f)
    want = gf.backward(b.x, b.wg[of], b.wu[of], b.dhw[:, of], "silu")
    within(b.dwgw[of], want, "dwg")
    within(b.dwuw[of], want, "dwu")
