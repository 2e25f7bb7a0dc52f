"""Performance cases of the eight-bit operators: tokens and activations held in 8 bits, the products that
read them, and the weight gradient from an 8-bit checkpoint.

Three kinds of call (``op``):

* ``keep``    an activation written to 8 bits and read back (sr_quantize8, sr_dequantize8), ``kind``
              "row" (one fp32 scale per token: the operands of the products) or "block" (a power of two
              per 32 channels: what a forward keeps for its backward);
* ``linear``  a linear layer on 8-bit integers: the tokens quantised by row (sr_quantize8), then the
              product with weights that were quantised once (sr_linear8), with bias and optional GELU;
* ``wgrad``   the weight and bias gradient of a linear layer from the 8-bit checkpoint of its input
              (sr_weight_grad8).

M is the number of tokens of the call (B x K), K the input and N the output channels.
"""
from __future__ import annotations

import math

import torch

own = False   # False: the plain forms in elementary torch operations; True: the library's calls


def _case(op, M, N, K, **kw):
    c = dict(op=op, M=M, N=N, K=K, dtype="bf16", kind="block", gelu=False)
    c.update(kw)
    return c


def listed():
    out = []

    def add(name, *a, **kw):
        out.append(dict(_case(*a, **kw), name=name))

    # what one block on a small grid keeps, in the fp32 storage mode
    add("keep_tiny_f32", "keep", 32, 0, 512, dtype="f32")
    # the MLP pre-activation of a block at 5.625 deg, eight samples of 128 routed tokens
    add("keep_5625", "keep", 1024, 0, 4096)
    # the MLP pre-activation of a dense block at 0.25 deg
    add("keep_025", "keep", 16200, 0, 4096)
    # the tokens of a dense block at 0.25 deg as operands of a product
    add("keep_rows_025", "keep", 16200, 0, 1024, kind="row")
    # one token through the first MLP product: latency
    add("linear_token", "linear", 1, 4096, 1024, gelu=True)
    # a forecast of one sample at 5.625 deg: the second MLP product on 128 routed tokens
    add("linear_5625", "linear", 128, 1024, 4096)
    # the fp32 mode of the width-256 forecaster on a ragged token count: the first MLP product
    add("linear_f32", "linear", 4083, 1024, 256, dtype="f32")
    # routed tokens at 0.25 deg: the output projection
    add("linear_routed_025", "linear", 4050, 1024, 1024)
    # a dense block at 0.25 deg: the first MLP product with its GELU
    add("linear_025", "linear", 16200, 4096, 1024, gelu=True)
    # the fp32 mode of the width-256 forecaster: gradient of the first MLP weight, ragged tokens
    add("wgrad_f32", "wgrad", 2013, 1024, 256, dtype="f32")
    # training at 5.625 deg: the second MLP weight
    add("wgrad_5625", "wgrad", 1024, 1024, 4096)
    # a dense block at 0.25 deg: the second MLP weight over all 16200 tokens
    add("wgrad_025", "wgrad", 16200, 1024, 4096)
    return out


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def channels():   # whole heads of 32, 64 or 128 channels, up to the widest MLP
        return 64 * log_int(1, 64)

    while True:
        op = rng.choice(["keep", "linear", "linear", "wgrad"])
        M, K = log_int(1, 16384), channels()
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if op == "keep":
            c = _case(op, M, 0, K, dtype=dtype, kind=rng.choice(["block", "row"]))
        elif op == "linear":   # outputs are block products or the forecaster's head (any multiple of 8)
            N = rng.choice([channels(), channels(), 8 * log_int(1, 512)])
            c = _case(op, M, N, K, dtype=dtype, gelu=rng.random() < 0.4)
        else:
            c = _case(op, M, rng.choice([channels(), channels(), 8 * log_int(1, 512)]), K, dtype=dtype)
        if K <= 4096 and M * K <= 16200 * 4096 and M * max(c["N"], 1) * K <= 16200 * 4096 * 1024:
            return c


# ------------------------------------------------------------------------------ inputs

BLOCK = 32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _tokens(gen, M, K):
    """Activations: unit normals, some channels several times larger than the rest, tokens of unequal size."""
    x = torch.randn((M, K), generator=gen, device="cuda")
    ch = torch.exp(0.5 * torch.randn((1, K), generator=gen, device="cuda"))
    tok = torch.exp(0.3 * torch.randn((M, 1), generator=gen, device="cuda"))
    return x.mul_(ch).mul_(tok)


def _plain_rows(x):
    """codes and scales of SR_Q8_ROW, in 64 bits next to the rounding borders."""
    amax = x.abs().amax(1, keepdim=True)
    t = x.double() * 127.0 / torch.where(amax > 0, amax, torch.ones_like(amax)).double()
    return torch.round(t).to(torch.int8), (amax / 127.0).float()


def _plain_blocks(x):
    """codes and exponents of SR_Q8_BLOCK."""
    b = x.view(x.shape[0], -1, BLOCK).double()
    m, e = torch.frexp(b.abs().amax(2, keepdim=True))
    e = torch.where(m > 127.0 / 128.0, e - 6, e - 7)
    e = torch.where(m == 0, torch.full_like(e, -126), e).clamp(-126, 121)
    q = torch.round(torch.ldexp(b, -e)).clamp_(-127, 127)
    return q.to(torch.int8).view(x.shape), e.squeeze(2)


def prepare(case, seed):
    c, gen = case, _gen(seed)
    M, N, K, dt = c["M"], c["N"], c["K"], _dtype(c)
    s = dict(c)
    empty = lambda shape, d: torch.empty(shape, dtype=d, device="cuda")  # noqa: E731
    x = _tokens(gen, M, K).to(dt)
    if c["op"] == "wgrad":   # the checkpoint that the forward wrote, and the gradient of the layer's output
        s["xq"], e = _plain_blocks(x.float())
        s["xe"] = (e + 127).to(torch.uint8)
        s["dy"] = (0.05 * _tokens(gen, M, N)).to(dt)
        s["dw"], s["db"] = empty((N, K), torch.float32), empty((N,), torch.float32)
        return s
    s["x"], s["xq"] = x, empty((M, K), torch.int8)
    s["xs"] = empty((M,), torch.float32) if c["op"] == "linear" or c["kind"] == "row" else empty((M, K // BLOCK), torch.uint8)
    if c["op"] == "keep":
        s["xhat"] = empty((M, K), dt)
        return s
    w = 0.02 * torch.randn((N, K), generator=gen, device="cuda")   # the weights, quantised by output channel
    s["wq"], ws = _plain_rows(w)
    s["ws"] = ws.view(N).contiguous()
    s["bias"] = (0.05 * torch.randn((N,), generator=gen, device="cuda")).to(dt)
    s["y"] = empty((M, N), dt)
    return s


# ------------------------------------------------------------------------------ one pass


def _run_plain(s):
    op, dt = s["op"], _dtype(s)
    if op == "keep":
        x = s["x"].float()
        if s["kind"] == "row":
            q, scale = _plain_rows(x)
            return {"xhat": (q.float() * scale).to(dt), "scale": scale.view(-1)}
        q, e = _plain_blocks(x)
        return {"xhat": torch.ldexp(q.view(*e.shape, BLOCK).float(), e.unsqueeze(2)).view(x.shape).to(dt)}
    if op == "linear":
        q, scale = _plain_rows(s["x"].float())
        y = torch.matmul(q.float(), s["wq"].float().t()) * scale * s["ws"] + s["bias"].float()
        if s["gelu"]:
            y = 0.5 * y * torch.erfc(y * -math.sqrt(0.5))
        return {"y": y.to(dt)}
    e = (s["xe"].int() - 127).unsqueeze(2)
    xhat = torch.ldexp(s["xq"].view(e.shape[0], -1, BLOCK).float(), e).view(s["xq"].shape)
    dy = s["dy"].float()
    return {"dw": torch.matmul(dy.t(), xhat), "db": dy.sum(0)}


def _run_own(s):
    from paper_2607_02829_amd import abi
    op, M, N, K = s["op"], s["M"], s["N"], s["K"]
    dt = abi.SR_BF16 if s["dtype"] == "bf16" else abi.SR_F32
    if op == "keep":
        kind = abi.SR_Q8_ROW if s["kind"] == "row" else abi.SR_Q8_BLOCK
        abi.sr_quantize8(kind, dt, M, K, s["x"], s["xq"], s["xs"])
        abi.sr_dequantize8(kind, dt, M, K, s["xq"], s["xs"], s["xhat"])
        return {"xhat": s["xhat"], "scale": s["xs"]} if s["kind"] == "row" else {"xhat": s["xhat"]}
    if op == "linear":
        abi.sr_quantize8(abi.SR_Q8_ROW, dt, M, K, s["x"], s["xq"], s["xs"])
        abi.sr_linear8(dt, abi.SR_ACT_GELU if s["gelu"] else abi.SR_ACT_NONE, M, N, K, s["xq"], s["xs"], s["wq"],
                       s["ws"], s["bias"], s["y"])
        return {"y": s["y"]}
    if "scratch" not in s:   # the workspace, which a training program keeps
        n = abi.sr_weight_grad8_scratch_bytes(dt, M, N, K)
        s["scratch"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    abi.sr_weight_grad8(dt, M, N, K, s["dy"], s["xq"], s["xe"], s["dw"], s["db"], s["scratch"])
    return {"dw": s["dw"], "db": s["db"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    M, N, K, e = case["M"], case["N"], case["K"], 2 if case["dtype"] == "bf16" else 4
    scales = 4 * M if case["op"] == "linear" or case["kind"] == "row" else M * K // BLOCK
    if case["op"] == "keep":   # read the values, write the codes; read the codes, write the values
        return {"bytes": 2 * (e * M * K + M * K + scales), "flops": 0}
    if case["op"] == "linear":
        return {"bytes": e * M * K + N * K + 4 * N + e * N + e * M * N, "flops": 2 * M * N * K}
    return {"bytes": e * M * N + M * K + M * K // BLOCK + 4 * N * K + 4 * N, "flops": 2 * M * N * K}


# ------------------------------------------------------------------------------ 64-bit results


def _nearest_even(t):
    """Integers nearest to t, halves to the even one."""
    f = torch.floor(t)
    d = t - f
    up = (d > 0.5) | ((d == 0.5) & (torch.remainder(f, 2.0) == 1.0))
    return f + up.to(t.dtype)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "wgrad":
        xhat = s["xq"].double() * torch.exp2(s["xe"].double() - 127.0).repeat_interleave(BLOCK, dim=1)
        dy = s["dy"].double()
        return {"dw": dy.t().contiguous() @ xhat, "db": dy.sum(0)}
    x = s["x"].double()
    if c["op"] == "keep" and c["kind"] == "block":
        top = x.abs().reshape(-1, BLOCK).amax(1, keepdim=True)
        e = torch.ceil(torch.log2((top / 127.0).clamp_min(2.0 ** -126)))
        e = e + (top > 127.0 * torch.exp2(e)).double()               # a border that the logarithm rounded over
        e = e - ((top <= 127.0 * torch.exp2(e - 1.0)) & (e > -126.0)).double()
        e = e.clamp(max=121.0)
        q = _nearest_even(x.reshape(-1, BLOCK) / torch.exp2(e)).clamp(-127.0, 127.0)
        return {"xhat": (q * torch.exp2(e)).reshape(x.shape)}
    top = x.abs().amax(1)
    q = _nearest_even(127.0 * x / torch.where(top > 0, top, 1.0)[:, None])
    scale = top / 127.0
    if c["op"] == "keep":
        return {"xhat": q * scale[:, None], "scale": scale}
    y = (q @ s["wq"].double().t().contiguous()) * scale[:, None] * s["ws"].double()[None, :] + s["bias"].double()[None, :]
    if c["gelu"]:   # y Phi(y)
        y = y * torch.special.ndtr(y)
    return {"y": y}
