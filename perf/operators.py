"""Cases of the gated feed-forward block and of dropout, their plain forms and their values in 64 bits.

``run`` with ``own`` false computes an operator with elementary torch operations in 32 bits, rounded once at the
end; with ``own`` true it makes the library's calls.  ``exact`` computes the same outputs in 64 bits.

The feed-forward block: h = D * act(x Wg^T) * (x Wu^T), with x [m, k], Wg and Wu [f, k] and D the dropout factor
of each element of h (1 without dropout).  Its backward pass takes x, Wg, Wu and dh and gives dx, dWg and dWu.
Dropout: y = residual + (kept ? x * scale : 0).  Whether element (row, col) is dropped is a function of (seed,
sequence, row, col): lane col % 8 (16 bits) of the Philox4x32-10 block with the counter (col // 8, row, sequence)
and the key seed, compared with round(65536 p).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _ffn(name, op, m, k, f, dtype, act, p=0.0, pad=0):
    # pad: x is a view of rows that are this many elements longer
    return {"name": name, "op": op, "m": m, "k": k, "f": f, "dtype": dtype, "act": act, "p": p, "pad": pad}


def _drop(name, op, rows, cols, dtype, p, residual):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "p": p, "residual": residual}


def listed():
    """Widths are powers of two with hidden widths of 8/3 of them, rounded up to 64, or odd sizes near them."""
    return [
        # one token of a small and of a large block: what a decoding step waits for
        _ffn("ffn token small", "ffn_forward", 1, 1024, 2752, "f16", "silu"),
        _ffn("ffn token", "ffn_forward", 1, 4096, 10944, "bf16", "silu"),
        # a decoding batch
        _ffn("ffn batch 24", "ffn_forward", 24, 2048, 5504, "bf16", "gelu"),
        # a short prompt on a block whose sizes are odd, rows of x inside a wider buffer
        _ffn("ffn ragged", "ffn_forward", 511, 1001, 2747, "f16", "relu", pad=6),
        # the forward pass of a training step, with dropout on the hidden map
        _ffn("ffn train", "ffn_forward", 8192, 4096, 10944, "bf16", "relu", p=0.1),
        # a model kept in single precision
        _ffn("ffn f32", "ffn_forward", 1000, 1024, 2752, "f32", "silu"),
        # backward: fine-tuning on a short text, odd sizes with dropout, and the training step
        _ffn("ffn backward short", "ffn_backward", 130, 1024, 2752, "bf16", "silu"),
        _ffn("ffn backward ragged", "ffn_backward", 777, 1003, 2731, "f16", "gelu", p=0.25),
        _ffn("ffn backward train", "ffn_backward", 8192, 4096, 10944, "bf16", "relu", p=0.1),
        # dropout of a small map, of a block's output onto its residual, and of a gradient of the shape of the
        # first convolution layer's map (64 x 64 x 224 x 224, the benchmark's tensor)
        _drop("dropout small", "dropout", 61, 1003, "f32", 0.5, False),
        _drop("dropout residual", "dropout", 8192, 4096, "bf16", 0.1, True),
        _drop("dropout gradient", "dropout_backward", 1, 205520896, "f32", 0.5, False),
    ]


def _log_between(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))


def _size(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm: an odd multiple of 64 or of 8, or odd."""
    unit = rng.choice((64, 64, 8, 1))
    n = max(lo, min(hi - unit, _log_between(rng, lo, hi))) // unit
    return unit * (n | 1)


def draw(rng):
    dtype = rng.choice(("bf16", "bf16", "f16", "f16", "f32"))
    p = rng.choice((0.0, 0.1, 0.25, 0.5))
    kind = rng.choice(("ffn_forward", "ffn_forward", "ffn_backward", "ffn_backward", "dropout", "dropout_backward"))
    if kind.startswith("ffn"):
        m, k, f = rng.choice((1, 2)) * (_log_between(rng, 1, 4000) | 1), _size(rng, 256, 4096), _size(rng, 512, 10944)
        # no ReLU gradient in 32 bits: near zero the sign of G, and with it a whole gradient, hangs on G's last bit
        acts = ("silu", "gelu") if (dtype, kind) == ("f32", "ffn_backward") else ("relu", "silu", "gelu")
        case = _ffn("", kind, m, k, f, dtype, rng.choice(acts), p, rng.choice((0, 0, 8, 3)))
    else:
        cols = _size(rng, 256, 16384)
        rows = _log_between(rng, 1, max(2, 100_000_000 // cols))
        case = _drop("", kind, rows, cols, dtype, p or 0.3, kind == "dropout" and rng.random() < 0.5)
    del case["name"]
    return case


def prepare(case, seed):
    """Rows of about unit variance, weights that keep it, and the small gradients of a mean loss."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(rows, cols, scale, pad=0):
        full = torch.randn(rows, cols + pad, generator=g, device="cuda").mul_(scale).to(dtype)
        return full[:, :cols]

    state = dict(case, seed=1_000_003 * seed + 17, sequence=(seed << 33) + 5,
                 result=torch.zeros(2, dtype=torch.int64).pin_memory())
    if case["op"].startswith("ffn"):
        m, k, f = case["m"], case["k"], case["f"]
        state["x"] = normal(m, k, 1.0, case["pad"])
        state["wg"], state["wu"] = normal(f, k, k ** -0.5), normal(f, k, k ** -0.5)
        if case["op"] == "ffn_backward":
            state["dh"] = normal(m, f, 0.01)
            state["dx"] = torch.empty(m, k, dtype=dtype, device="cuda")
            state["dwg"], state["dwu"] = (torch.empty(f, k, dtype=dtype, device="cuda") for _ in range(2))
        else:
            state["h"] = torch.empty(m, f, dtype=dtype, device="cuda")
    else:
        state["x"] = normal(case["rows"], case["cols"], 1.0 if case["op"] == "dropout" else 0.01)
        state["residual"] = normal(case["rows"], case["cols"], 1.0) if case["residual"] else None
        state["y"] = torch.empty(case["rows"], case["cols"], dtype=dtype, device="cuda")
    return state


# ---- plain forms -------------------------------------------------------------------------------------------

def _mul_hi_lo(a, m):
    """High and low words of the product of 32-bit a (held in 64) and the constant m, by 16-bit halves of m."""
    low, high = a * (m & 0xffff), a * (m >> 16)
    return (high + (low >> 16)) >> 16, (low + ((high & 0xffff) << 16)) & 0xffffffff


def _plain_keep(rows, cols, p, seed, sequence):
    """Truth values [rows, cols]: which elements dropout keeps."""
    blocks = (cols + 7) // 8
    c0 = torch.arange(blocks, device="cuda").repeat(rows, 1)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, blocks)
    c2 = torch.full_like(c0, sequence & 0xffffffff)
    c3 = torch.full_like(c0, (sequence >> 32) & 0xffffffff)
    k0, k1 = seed & 0xffffffff, (seed >> 32) & 0xffffffff
    for _ in range(10):     # the generator's ten rounds
        h0, l0 = _mul_hi_lo(c0, 0xD2511F53)
        h1, l1 = _mul_hi_lo(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    words = torch.stack((c0, c1, c2, c3), dim=-1)
    lanes = torch.stack((words & 0xffff, words >> 16), dim=-1).reshape(rows, 8 * blocks)[:, :cols]
    return lanes >= round(p * 65536)


def _plain_drop(x, keep, p):
    dropped = round(p * 65536)
    scale = 65536.0 / (65536 - dropped) if dropped < 65536 else 0.0
    return torch.where(keep, x * scale, torch.zeros((), device=x.device))


def _plain_act(g, act):
    """act(g) and its derivative."""
    if act == "relu":
        return torch.clamp(g, min=0.0), (g > 0).float()
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain(s):
    dtype = DTYPES[s["dtype"]]
    p, seed, sequence = s["p"], s["seed"], s["sequence"]
    if s["op"].startswith("dropout"):
        y = _plain_drop(s["x"].float(), _plain_keep(s["rows"], s["cols"], p, seed, sequence), p)
        return (y if s["residual"] is None else s["residual"].float() + y).to(dtype)
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    a, da = _plain_act(g, s["act"])
    keep = _plain_keep(s["m"], s["f"], p, seed, sequence) if p else None
    if s["op"] == "ffn_forward":
        h = a * u
        return (h if keep is None else _plain_drop(h, keep, p)).to(dtype)
    e = s["dh"].float()
    e = e if keep is None else _plain_drop(e, keep, p)
    du, dg = e * a, e * u * da
    return {"dx": (dg @ wg + du @ wu).to(dtype), "dwg": (dg.t() @ x).to(dtype), "dwu": (du.t() @ x).to(dtype)}


# ---- the library's calls -----------------------------------------------------------------------------------

def _library(s):
    from paper_1705_01626_b200 import binding as B
    stream = torch.cuda.current_stream().cuda_stream
    if s["op"].startswith("dropout"):
        code = {"f32": B.F32, "f16": B.F16, "bf16": B.BF16}[s["dtype"]]
        x, y, cols = s["x"], s["y"], s["cols"]
        if s["op"] == "dropout":
            r = s["residual"]
            st = B.cdma_dropout(x.data_ptr(), x.stride(0), r.data_ptr() if r is not None else 0, cols, s["rows"], cols,
                                code, s["p"], s["seed"], s["sequence"], y.data_ptr(), cols, stream)
        else:
            st = B.cdma_dropout_backward(x.data_ptr(), x.stride(0), s["rows"], cols, code, s["p"], s["seed"],
                                         s["sequence"], y.data_ptr(), cols, stream)
        if st:
            raise B.CdmaError(st, s["op"])
        return y
    backward = s["op"] == "ffn_backward"
    if "plan" not in s:         # a program keeps its descriptor and its workspace
        s["plan"] = B.cdma_gated_ffn_desc(
            m=s["m"], k=s["k"], f=s["f"], ld_x=s["x"].stride(0), dtype={"f32": B.F32, "f16": B.F16, "bf16": B.BF16}[s["dtype"]],
            activation={"relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}[s["act"]],
            dropout_p=s["p"], dropout_seed=s["seed"], dropout_sequence=s["sequence"])
        s["ws"] = torch.empty(B.cdma_gated_ffn_workspace_bytes(s["plan"], int(backward)), dtype=torch.uint8, device="cuda")
    ws = s["ws"]
    if backward:
        st = B.cdma_gated_ffn_backward_async(s["plan"], s["x"].data_ptr(), s["wg"].data_ptr(), s["wu"].data_ptr(),
                                             s["dh"].data_ptr(), s["dx"].data_ptr(), s["dwg"].data_ptr(), s["dwu"].data_ptr(),
                                             ws.data_ptr(), ws.numel(), stream, s["result"].data_ptr())
        out = {"dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"]}
    else:
        st = B.cdma_gated_ffn_forward_async(s["plan"], s["x"].data_ptr(), s["wg"].data_ptr(), s["wu"].data_ptr(),
                                            s["h"].data_ptr(), ws.data_ptr(), ws.numel(), stream, s["result"].data_ptr())
        out = s["h"]
    if st:
        raise B.CdmaError(st, s["op"])
    return out


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("dropout"):
        n = case["rows"] * case["cols"]
        return {"bytes": size * n * (3 if case["residual"] else 2), "flops": 0}
    m, k, f = case["m"], case["k"], case["f"]
    if case["op"] == "ffn_forward":
        return {"bytes": size * (m * k + 2 * f * k + m * f), "flops": 4 * m * k * f}
    return {"bytes": size * (2 * m * k + 4 * f * k + m * f), "flops": 12 * m * k * f}


# ---- the same in 64 bits -----------------------------------------------------------------------------------

def _exact_factor(rows, cols, p, seed, sequence):
    """The dropout factor of each element (0 or 65536 / (65536 - T)), by numpy's unsigned 64-bit products."""
    threshold, word = round(p * 65536), np.uint64(0xffffffff)
    blocks = -(-cols // 8)
    out = torch.empty(rows, cols, dtype=torch.float64, device="cuda")
    lines = max(1, (1 << 22) // blocks)
    wide = 1 << 22
    for r in range(0, rows, lines):
        for b in range(0, blocks, wide):
            row, col = np.meshgrid(np.arange(r, min(rows, r + lines), dtype=np.uint64),
                                   np.arange(b, min(blocks, b + wide), dtype=np.uint64), indexing="ij")
            x = [col, row, np.full_like(col, sequence & 0xffffffff), np.full_like(col, (sequence >> 32) & 0xffffffff)]
            key = [seed & 0xffffffff, (seed >> 32) & 0xffffffff]
            for _ in range(10):
                p0, p1 = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
                x = [(p1 >> np.uint64(32)) ^ x[1] ^ np.uint64(key[0]), p1 & word,
                     (p0 >> np.uint64(32)) ^ x[3] ^ np.uint64(key[1]), p0 & word]
                key = [(key[0] + 0x9E3779B9) & 0xffffffff, (key[1] + 0xBB67AE85) & 0xffffffff]
            lanes = np.stack([v.astype("<u4") for v in x], axis=-1).view("<u2").reshape(row.shape[0], -1)
            kept = torch.from_numpy(lanes >= threshold)
            there = out[r:r + lines, 8 * b:8 * (b + wide)]
            there.copy_(kept[:, :there.shape[1]])
    return out * (65536 / (65536 - threshold) if threshold < 65536 else 0.0)


def exact(case, seed):
    s = prepare(case, seed)
    p = case["p"]
    if case["op"].startswith("dropout"):
        y = _exact_factor(case["rows"], case["cols"], p, s["seed"], s["sequence"]).mul_(s["x"])
        return y if s["residual"] is None else y.add_(s["residual"])
    x, wg, wu = (s[n].double() for n in ("x", "wg", "wu"))
    g = torch.einsum("mk,fk->mf", x, wg)
    u = torch.einsum("mk,fk->mf", x, wu)
    if case["act"] == "relu":
        a, slope = g.relu(), torch.heaviside(g, torch.zeros_like(g[:1, :1]))
    elif case["act"] == "silu":
        a, slope = g * g.sigmoid(), g.sigmoid() + g * g.sigmoid() * (-g).sigmoid()
    else:
        phi = torch.special.ndtr(g)
        a, slope = g * phi, phi + g * (-g.square() / 2).exp() / math.sqrt(2 * math.pi)
    factor = _exact_factor(case["m"], case["f"], p, s["seed"], s["sequence"]) if p else torch.ones((), dtype=torch.float64, device="cuda")
    if case["op"] == "ffn_forward":
        return factor * a * u
    e = factor * s["dh"].double()
    dg, du = e * u * slope, e * a
    return {"dx": torch.einsum("mf,fk->mk", dg, wg) + torch.einsum("mf,fk->mk", du, wu),
            "dwg": torch.einsum("mf,mk->fk", dg, x), "dwu": torch.einsum("mf,mk->fk", du, x)}
