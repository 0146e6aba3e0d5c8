"""The operators around the DP weight gradient that this library is timed on: the other layers of a transformer block that
is trained under per-layer DP-SGD, each in its plain form and as the library's call.

A case names an operator and a problem:
  op      "linear"      flashdp_linear_forward: Y = act(X W^T + bias) + residual, the sum Z in front of the activation kept
                        on demand
          "activation"  flashdp_activation_dp_grad: dZ = dY act'(Z) and the bias's clipped, noised gradient
          "layernorm"   flashdp_layernorm_forward
          "layernorm_train"  the same and flashdp_layernorm_dp_grad: dX and the clipped, noised gradient of weight and bias
          "checkpoint"  flashdp_checkpoint8_pack and _unpack: an activation to 8 bits and back
          "checkpoint_grad"  flashdp_block_dp_grad_checkpoint8: the weight's clipped, noised gradient from an 8-bit activation
  dtype   storage of activations, weights and their gradients: "bf16", "f16" or "fp32"
  B, T    samples and tokens per sample (the forward products and 8-bit checkpoints only see B * T rows)
  d_in, d_out   features (normalisations and checkpoints have d_in only, activations d_out only)
  act     "none", "relu", "gelu", "gelu_tanh" or "silu"
  keep    how Z is kept: "none", "dtype" or "8bit"
  bias, residual   whether a linear layer has them
  C, sigma   clipping threshold and noise multiplier of the gradients

8-bit checkpoints: blocks of 32 consecutive features of a row share an exponent e; an element is q 2^e with q an
integer from -127 to 127.  With m the largest magnitude of a block, e = floor(log2 m) - 6, at least -126 (fp16: -24), and
q = round(x 2^-e), ties to even, cut to that range.  The buffer holds the q of all rows (int8, rows * d_in, padded to a
multiple of 16 bytes), then the e + 127 (uint8, rows * ceil(d_in / 32)).

The noise of a vector of parameters is the field of the weights with 1 (bias) or 2 (normalisations) as last counter word.

Sizes are those of this repository's workloads (GPT-2 and Llama layers) and generic ones.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "fp32": 4}
BLOCK = 32
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
BIAS_FIELD, NORM_FIELD = 1, 2
EPS = 1e-5


def _case(name, op, dtype, B, T, d_in=0, d_out=0, act="none", keep="none", bias=False, residual=False, C=1.0, sigma=0.0):
    return dict(name=name, op=op, dtype=dtype, B=B, T=T, d_in=d_in, d_out=d_out, act=act, keep=keep, bias=bias, residual=residual,
                C=C, sigma=sigma)


def listed():
    return [
        # one new token through the output projection of an attention block, added to the residual stream: W is read once
        _case("linear_token", "linear", "bf16", 1, 1, 4096, 4096, residual=True),
        # the up-projection of a GPT-2 MLP in training: bias and GELU, Z kept in 8 bits for the backward pass
        _case("linear_gpt2_up_8bit", "linear", "bf16", 8, 1024, 768, 3072, act="gelu_tanh", keep="8bit", bias=True),
        # the output layer over GPT-2's vocabulary for the last token of eight sequences: an odd number of features
        _case("linear_vocab_odd", "linear", "f16", 8, 1, 768, 50257),
        # a Llama-13B MLP projection with its activation, Z kept as it is
        _case("linear_llama13b_gate", "linear", "bf16", 4, 2048, 5120, 13824, act="silu", keep="dtype"),
        # single precision: an attention projection with bias and residual
        _case("linear_fp32", "linear", "fp32", 1, 2048, 4096, 4096, bias=True, residual=True),
        # rows without a sequence (T = 1), the many-small-samples end of DP-SGD: a hidden layer of a classifier
        _case("activation_rows", "activation", "fp32", 256, 1, d_out=512, act="relu", keep="dtype", sigma=1.0),
        # the backward pass of the GPT-2 up-projection's bias and GELU, from Z in 8 bits
        _case("activation_gpt2_8bit", "activation", "bf16", 8, 1024, d_out=3072, act="gelu_tanh", keep="8bit", sigma=1.0),
        # one token of a generating model: latency
        _case("layernorm_token", "layernorm", "bf16", 1, 1, 5120),
        # the normalisations of a GPT-2 and of a Llama-13B block in training, forward and backward; tokens no tile divides in the first
        _case("layernorm_gpt2", "layernorm_train", "f16", 8, 1021, 768, sigma=0.8),
        _case("layernorm_13b", "layernorm_train", "bf16", 8, 2048, 5120, sigma=1.0),
        # the input of a Llama-13B block's projections, kept in 8 bits between forward and backward pass
        _case("checkpoint_13b", "checkpoint", "bf16", 8, 2048, 5120),
        # the Llama-7B attention projection's weight gradient from such a checkpoint
        _case("checkpoint_grad_7b", "checkpoint_grad", "bf16", 4, 2048, 4096, 4096, sigma=0.8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: operator, type and sizes independent of each other, sizes log-uniform, cut down until it costs no more
    than the Llama-13B projection."""
    op = rng.choice(["linear", "linear", "linear", "activation", "activation", "layernorm", "layernorm_train", "layernorm_train",
                     "checkpoint", "checkpoint_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "fp32"])
    align = rng.choice([1, 8, 8, 64])
    T = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 64, 2048), _log_int(rng, 512, 2048)])
    B = _log_int(rng, 1, 256 if T <= 16 else 64 if T <= 256 else 16)
    d_in, d_out = (max(align, _log_int(rng, 24, 13824) // align * align) for _ in range(2))
    act = rng.choice(ACTS)
    c = _case("", op, dtype, B, T, d_in, d_out, act=act, keep=rng.choice(["none", "dtype", "8bit"]), bias=rng.random() < 0.5,
              residual=rng.random() < 0.5, C=rng.choice([0.1, 1.0, 10.0]), sigma=rng.choice([0.0, 0.5, 1.0]))
    c.pop("name")
    if op == "activation":
        c["d_in"] = 0
        c["keep"] = rng.choice(["dtype", "8bit"]) if act != "none" else "none"
        c["bias"] = True
    elif op != "linear":
        c.update(act="none", keep="none", bias=False, residual=False)
        if op != "checkpoint_grad":
            c["d_out"] = 0
    if op in ("linear", "layernorm", "checkpoint"):
        c.update(C=1.0, sigma=0.0)
    if op == "linear" and dtype == "fp32" and c["keep"] == "8bit":
        # two correct sums that lie on either side of a border between 8-bit values are a step apart, far more than single
        # precision tells apart
        c["keep"] = "dtype"

    def too_much():
        rows, p, d = c["B"] * c["T"], max(1, c["d_in"]), max(1, c["d_out"])
        return 2.0 * rows * p * d > 1.1e12 or rows * max(p, d) > 1.1e8 or (op == "checkpoint_grad" and (c["B"] * p * d > 1.2e8 or rows * p * d > 1.4e11))

    while too_much():
        k = rng.choice([v for v in ("B", "d_in", "d_out") if c[v] > 1])
        c[k] = max(align if k != "B" else 1, c[k] * 2 // 3 // (align if k != "B" else 1) * (align if k != "B" else 1))
    return c


# ---- inputs ----------------------------------------------------------------------------------------

def _randn(gen, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEVICE) * scale).to(dtype)


def _gradient(gen, B, T, d, dtype):
    """Output gradients: small, with a scale of its own for each sample, so that norms spread over two decades."""
    scale = 1e-2 * 10.0 ** (2.0 * torch.rand((B, 1, 1), generator=gen, device=DEVICE) - 1.0)
    return (torch.randn((B, T, d), generator=gen, device=DEVICE) * scale).to(dtype)


def _stream(gen, rows, d, dtype):
    """Activations as a normalisation meets them: a residual stream with an offset and a few large features."""
    x = torch.randn((rows, d), generator=gen, device=DEVICE)
    feature = torch.randn((d,), generator=gen, device=DEVICE)
    return (x * (1.0 + 8.0 * (feature > 2.2)) + 0.3 * feature).to(dtype)


def _exponents(blocks, least):
    """Biased exponents of blocks (..., 32) of finite values."""
    top = blocks.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top)[1] - 7).clamp(min=least)      # frexp: top = f 2^e with 1/2 <= f < 1
    return torch.where(top > 0, e, torch.full_like(e, least))


def _blocks(x):
    rows, d = x.shape
    pad = -d % BLOCK
    return torch.nn.functional.pad(x, (0, pad)).reshape(rows, (d + pad) // BLOCK, BLOCK)


def _least(dtype):
    return -24 if dtype in ("f16", torch.float16) else -126


def _power(e):
    """2^e in fp32 from its bits, -126 <= e <= 127."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _quantised(x32, least):
    """(q, e) of the 8-bit form of fp32 rows."""
    b = _blocks(x32)
    e = _exponents(b, least)
    q = (b * _power(-e)).round().clamp(-127, 127)
    return q, e


def _values(q, e, d):
    return (q * _power(e)).reshape(q.shape[0], -1)[:, :d]


def _packed(x):
    """The buffer that an 8-bit checkpoint of x (rows, d) is."""
    rows, d = x.shape
    q, e = _quantised(x.float(), _least(x.dtype))
    head = (rows * d + 15) // 16 * 16
    nb = e.shape[1]
    buf = torch.zeros((head + rows * nb,), dtype=torch.uint8, device=x.device)
    buf[:rows * d] = q.reshape(rows, -1)[:, :d].to(torch.int8).reshape(-1).view(torch.uint8)
    buf[head:] = (e.reshape(-1) + 127).to(torch.uint8)
    return buf


def _unpacked(buf, rows, d):
    """fp32 values of such a buffer."""
    nb, head = -(-d // BLOCK), (rows * d + 15) // 16 * 16
    q = _blocks(buf[:rows * d].view(torch.int8).reshape(rows, d).float())
    e = buf[head:head + rows * nb].to(torch.int32).reshape(rows, nb, 1) - 127
    return _values(q, e, d)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    op, dt = case["op"], _TORCH[case["dtype"]]
    B, T, p, d = case["B"], case["T"], case["d_in"], case["d_out"]
    rows = B * T
    s = dict(case)
    s.update(rows=rows, dt=dt, seed=1 + seed % (1 << 30), layer=seed % 97)
    new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device=DEVICE)   # noqa: E731
    if op == "linear":
        s["x"] = _randn(gen, (rows, p), dt)
        s["w"] = _randn(gen, (d, p), dt, p ** -0.5)
        s["b"] = _randn(gen, (d,), dt, 0.1) if case["bias"] else None
        s["r"] = _randn(gen, (rows, d), dt) if case["residual"] else None
        s["y"] = new(rows, d)
        if case["keep"] != "none":
            s["z"] = new(rows, d)       # where Z is kept in 8 bits, its values are brought back here
        if case["keep"] == "8bit":
            s["z8"] = new((rows * d + 15) // 16 * 16 + rows * -(-d // BLOCK), dtype=torch.uint8)
    elif op == "activation":
        s["dy"] = _gradient(gen, B, T, d, dt)
        if case["keep"] != "none":
            z = _randn(gen, (rows, d), dt, 1.5)
            s["z"] = _packed(z) if case["keep"] == "8bit" else z
            s["dz"] = new(B, T, d)
        s["g"], s["n"] = new(d, dtype=torch.float32), new(B, dtype=torch.float32)
    elif op in ("layernorm", "layernorm_train"):
        s["x"] = _stream(gen, rows, p, dt)
        s["w"] = (1.0 + 0.1 * torch.randn((p,), generator=gen, device=DEVICE)).to(dt)
        s["b"] = _randn(gen, (p,), dt, 0.1)
        s["y"], s["mean"], s["rstd"] = new(rows, p), new(rows, dtype=torch.float32), new(rows, dtype=torch.float32)
        if op == "layernorm_train":
            s["dy"] = _gradient(gen, B, T, p, dt)
            s["dx"], s["g"], s["n"] = new(B, T, p), new(2, p, dtype=torch.float32), new(B, dtype=torch.float32)
    elif op == "checkpoint":
        s["x"] = _stream(gen, rows, p, dt)
        s["y"] = new(rows, p)
        s["x8"] = new((rows * p + 15) // 16 * 16 + rows * -(-p // BLOCK), dtype=torch.uint8)
    else:
        s["x8"] = _packed(_stream(gen, rows, p, dt))
        s["dy"] = _gradient(gen, B, T, d, dt)
        s["g"], s["n"] = new(d, p, dtype=torch.float32), new(B, dtype=torch.float32)
    return s


# ---- plain forms -----------------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return z * 0.5 * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2.0 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * k * (1.0 + 3.0 * 0.044715 * z * z)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _noise(seed, layer, field, n):
    """n values of the noise field: ten rounds of Philox4x32 in 64-bit integers, then Box-Muller in 64 bits."""
    low = 0xFFFFFFFF
    g = torch.arange((n + 3) // 4, dtype=torch.int64, device=DEVICE)
    c0, c1 = g & low, g >> 32
    c2, c3 = torch.full_like(g, layer), torch.full_like(g, field)
    k0, k1 = seed & low, seed >> 32

    def product(m, c):      # high and low halves of a 32 x 32 bit product
        t = m * (c & 0xFFFF)
        u = m * (c >> 16) + (t >> 16)
        return u >> 16, ((u & 0xFFFF) << 16) | (t & 0xFFFF)

    for _ in range(10):
        h0, l0 = product(0xD2511F53, c0)
        h1, l1 = product(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    u = ((torch.stack((c0, c1, c2, c3), 1) >> 8).double() + 0.5) * 2.0 ** -24
    radius, angle = torch.sqrt(-2.0 * torch.log(u[:, 0::2])), 2.0 * math.pi * u[:, 1::2]
    return torch.stack((radius * torch.cos(angle), radius * torch.sin(angle)), 2).reshape(-1)[:n].float()


def _clipped(G, s, field):
    """sum_i G_i / max(1, |G_i| / C) + sigma C z and the norms, of per-sample gradients G (B, ...) in 32 bits."""
    B = G.shape[0]
    norms = G.reshape(B, -1).square().sum(1, dtype=torch.float64).sqrt()
    c = (1.0 / (norms / s["C"]).clamp(min=1.0)).float()
    out = (G * c.reshape(-1, *(1,) * (G.dim() - 1))).sum(0)
    if s["sigma"] > 0:
        out = out + s["sigma"] * s["C"] * _noise(s["seed"], s["layer"], field, out.numel()).reshape(out.shape)
    return out, norms.float()


def _plain(s):
    op, dt, rows, p, d = s["op"], s["dt"], s["rows"], s["d_in"], s["d_out"]
    if op == "linear":
        z = s["x"].float() @ s["w"].float().t()
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _act(z, s["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        out = dict(y=y.to(dt))
        if s["keep"] == "dtype":
            out["z"] = z.to(dt)
        elif s["keep"] == "8bit":
            out["z"] = _values(*_quantised(z, _least(dt)), d).to(dt)
        return out
    if op == "activation":
        dz = s["dy"].float()
        out = {}
        if s["keep"] != "none":
            z = _unpacked(s["z"], rows, d) if s["keep"] == "8bit" else s["z"].float()
            dz = dz * _slope(z, s["act"]).reshape(dz.shape)
            out["dz"] = dz.to(dt)
        out["g"], out["n"] = _clipped(dz.sum(1), s, BIAS_FIELD)
        return out
    if op in ("layernorm", "layernorm_train"):
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        rstd = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        xh, w = (x - mean) * rstd, s["w"].float()
        out = dict(y=(xh * w + s["b"].float()).to(dt), mean=mean.reshape(-1), rstd=rstd.reshape(-1))
        if op == "layernorm_train":
            dy = s["dy"].float()
            a = dy.reshape(rows, p) * w
            dx = rstd * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
            out["dx"] = dx.to(dt).reshape(dy.shape)
            out["g"], out["n"] = _clipped(torch.stack(((dy * xh.reshape(dy.shape)).sum(1), dy.sum(1)), 1), s, NORM_FIELD)
        return out
    if op == "checkpoint":
        return _values(*_quantised(s["x"].float(), _least(dt)), p).to(dt)
    x = _unpacked(s["x8"], rows, p).reshape(s["B"], s["T"], p)
    g, n = _clipped(s["dy"].float().transpose(1, 2).contiguous() @ x, s, 0)
    return dict(g=g, n=n)


# ---- the library's calls ---------------------------------------------------------------------------

def _own(s):
    import paper_2507_01154_amd as F
    op, B, T, p, d, rows = s["op"], s["B"], s["T"], s["d_in"], s["d_out"], s["rows"]
    code = {"bf16": F.BF16, "f16": F.F16, "fp32": F.F32}[s["dtype"]]
    if op == "linear":
        z = {"none": None, "dtype": s.get("z"), "8bit": s.get("z8")}[s["keep"]]
        F.flashdp_linear_forward(s["x"], s["w"], s["b"], s["r"], rows, p, d, code, s["act"], s["y"], z, s["keep"] == "8bit")
        if s["keep"] == "8bit":
            F.flashdp_checkpoint8_unpack(s["z8"], rows, d, code, s["z"])
        return dict(y=s["y"]) if z is None else dict(y=s["y"], z=s["z"])
    if op == "activation":
        F.flashdp_activation_dp_grad(s["dy"], s.get("z"), s["keep"] == "8bit", B, T, d, code, s["act"], s["C"], s["sigma"], s["seed"], s["layer"],
                                     s.get("dz"), s["g"], s["n"])
        return dict(g=s["g"], n=s["n"]) if s["keep"] == "none" else dict(dz=s["dz"], g=s["g"], n=s["n"])
    if op in ("layernorm", "layernorm_train"):
        F.flashdp_layernorm_forward(s["x"], s["w"], s["b"], rows, p, code, EPS, s["y"], s["mean"], s["rstd"])
        out = dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
        if op == "layernorm_train":
            F.flashdp_layernorm_dp_grad(s["x"], s["dy"], s["w"], s["mean"], s["rstd"], B, T, p, code, s["C"], s["sigma"], s["seed"], s["layer"],
                                        s["dx"], s["g"], s["n"])
            out.update(dx=s["dx"], g=s["g"], n=s["n"])
        return out
    if op == "checkpoint":
        F.flashdp_checkpoint8_pack(s["x"], rows, p, code, s["x8"])
        F.flashdp_checkpoint8_unpack(s["x8"], rows, p, code, s["y"])
        return s["y"]
    layer = dict(X=s["x8"], dY=s["dy"], d_in=p, d_out=d, C=s["C"], sigma=s["sigma"], seed=s["seed"], layer=s["layer"], out_grad=s["g"], out_norms=s["n"])
    # whoever keeps activations in 8 bits is short of memory: the schedule that parks no per-sample gradients
    F.flashdp_block_dp_grad_checkpoint8([layer], B, T, code, "twopass")
    return dict(g=s["g"], n=s["n"])


def run(state):
    return _own(state) if own else _plain(state)


# ---- work and definition ---------------------------------------------------------------------------

def work(case):
    """Every operand read once and every result written once; one product per linear layer or weight gradient."""
    op, e, B, rows, p, d = case["op"], _BYTES[case["dtype"]], case["B"], case["B"] * case["T"], case["d_in"], case["d_out"]
    eight = lambda n: 1.0 + 1.0 / BLOCK if n else 0.0     # noqa: E731  bytes an element in 8 bits takes
    if op == "linear":
        z = {"none": 0.0, "dtype": float(e), "8bit": 2 * eight(1) + e}[case["keep"]]    # 8 bits: written, read back and returned
        return {"bytes": e * (rows * p + d * p + d * case["bias"] + rows * d * (1.0 + case["residual"])) + rows * d * z,
                "flops": 2.0 * rows * p * d}
    if op == "activation":
        z = {"none": 0.0, "dtype": 2.0 * e, "8bit": eight(1) + e}[case["keep"]]         # Z in, dZ out
        return {"bytes": rows * d * (e + z) + 4.0 * d + 4.0 * B, "flops": 10.0 * rows * d}
    if op == "layernorm":
        return {"bytes": 2.0 * e * rows * p + 2.0 * e * p + 8.0 * rows, "flops": 8.0 * rows * p}
    if op == "layernorm_train":
        return {"bytes": 5.0 * e * rows * p + 3.0 * e * p + 16.0 * rows + 8.0 * p + 4.0 * B, "flops": 20.0 * rows * p}
    if op == "checkpoint":
        return {"bytes": rows * p * 2.0 * (e + eight(1)), "flops": 4.0 * rows * p}
    return {"bytes": rows * (p * eight(1) + e * d) + 4.0 * p * d + 4.0 * B, "flops": 2.0 * rows * p * d}


def _field64(seed, layer, field, n):
    """The noise field again, in numpy's unsigned integers."""
    g = np.arange((n + 3) // 4, dtype=np.uint64)
    word = np.uint64(0xFFFFFFFF)
    c = [g & word, g >> np.uint64(32), np.full_like(g, layer), np.full_like(g, field)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), b & word, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), a & word]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    u = [((w >> np.uint64(8)).astype(np.float64) + 0.5) / 2.0 ** 24 for w in c]
    z = np.empty((g.size, 4))
    for k in (0, 2):
        r = np.sqrt(-2.0 * np.log(u[k]))
        z[:, k], z[:, k + 1] = r * np.cos(2.0 * np.pi * u[k + 1]), r * np.sin(2.0 * np.pi * u[k + 1])
    return torch.from_numpy(z.reshape(-1)[:n]).to(DEVICE)


def _sum64(per_sample, s, field):
    """Clip, add up, add noise, one sample after the other."""
    total, norms = None, []
    for G in per_sample:
        norms.append(float(G.square().sum().sqrt()))
        G = G / max(1.0, norms[-1] / s["C"])
        total = G if total is None else total + G
    if s["sigma"] > 0:
        total = total + s["sigma"] * s["C"] * _field64(s["seed"], s["layer"], field, total.numel()).reshape(total.shape)
    return total, torch.tensor(norms, dtype=torch.float64)


def _act64(z, act):
    """(value, slope) by erfc and logistic functions."""
    one = torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, 0 * one), torch.where(z > 0, one, 0 * one)
    if act == "gelu":
        half = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return z * half, half + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act in ("gelu_tanh", "silu"):
        k = 2.0 * math.sqrt(2.0 / math.pi) if act == "gelu_tanh" else 1.0
        u = k * (z + 0.044715 * z ** 3) if act == "gelu_tanh" else z
        du = k * (1 + 3 * 0.044715 * z * z) if act == "gelu_tanh" else one
        s = torch.sigmoid(u)
        return z * s, s + z * s * torch.sigmoid(-u) * du
    return z, one


def _eight64(x, f16):
    """The values that 8 bits hold of x (rows, d), in 64 bits."""
    rows, d = x.shape
    out = torch.zeros((rows, -(-d // BLOCK) * BLOCK), dtype=torch.float64, device=x.device)
    out[:, :d] = x
    out = out.view(rows, -1, BLOCK)
    top = out.abs().max(-1, keepdim=True).values
    least = -24 if f16 else -126
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140))) - 6
    e = e + (top >= 2.0 ** (e + 7)).double() - (top < 2.0 ** (e + 6)).double()     # the logarithm may be off by one at a power of two
    step = ((e.clamp(min=least).long() + 1023) << 52).view(torch.float64)     # 2^e to the bit: ties of x / step stay ties
    return (torch.clamp(torch.round(out / step), -127, 127) * step).reshape(rows, -1)[:, :d]


def _from8(buf, rows, d):
    """The values of a checkpoint's buffer in 64 bits."""
    bytes_ = buf.cpu().numpy()
    nb = -(-d // BLOCK)
    q = bytes_[:rows * d].view(np.int8).reshape(rows, d).astype(np.float64)
    e = bytes_[bytes_.size - rows * nb:].reshape(rows, nb).astype(np.int64) - 127
    return torch.from_numpy(np.ldexp(q, np.repeat(e, BLOCK, axis=1)[:, :d])).to(DEVICE)


def exact(case, seed):
    s = prepare(case, seed)
    op, B, T, p, d, rows = s["op"], s["B"], s["T"], s["d_in"], s["d_out"], s["rows"]
    f16 = s["dtype"] == "f16"
    if op == "linear":
        z = torch.matmul(s["x"].double(), s["w"].double().T)
        if s["b"] is not None:
            z += s["b"].double()
        y = _act64(z, s["act"])[0]
        if s["r"] is not None:
            y = y + s["r"].double()
        kept = {"none": None, "dtype": z, "8bit": _eight64(z, f16) if s["keep"] == "8bit" else None}[s["keep"]]
        return dict(y=y) if kept is None else dict(y=y, z=kept)
    if op == "activation":
        dz, out = s["dy"].double(), {}
        if s["keep"] != "none":
            z = _from8(s["z"], rows, d) if s["keep"] == "8bit" else s["z"].double()
            dz = dz * _act64(z, s["act"])[1].view_as(dz)
            out["dz"] = dz
        out["g"], out["n"] = _sum64((dz[i].sum(0) for i in range(B)), s, BIAS_FIELD)
        return out
    if op in ("layernorm", "layernorm_train"):
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS) ** -0.5
        xh = (x - mean[:, None]) * rstd[:, None]
        out = dict(y=xh * s["w"].double() + s["b"].double(), mean=mean, rstd=rstd)
        if op == "layernorm_train":
            dy = s["dy"].double().view(rows, p)
            a = dy * s["w"].double()
            out["dx"] = ((a - (a.sum(1) / p)[:, None] - xh * ((a * xh).sum(1) / p)[:, None]) * rstd[:, None]).view(B, T, p)
            both = lambda i: torch.stack(((dy * xh)[i * T:(i + 1) * T].sum(0), dy[i * T:(i + 1) * T].sum(0)))   # noqa: E731
            out["g"], out["n"] = _sum64((both(i) for i in range(B)), s, NORM_FIELD)
        return out
    if op == "checkpoint":
        return _eight64(s["x"].double(), f16)
    x, dy = _from8(s["x8"], rows, p).view(B, T, p), s["dy"].double()
    g, n = _sum64((torch.matmul(dy[i].T.contiguous(), x[i]) for i in range(B)), s, 0)
    return dict(g=g, n=n)
