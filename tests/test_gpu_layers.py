"""The layers around the weight gradient against their definitions in 64 bits on the CPU: forward product with epilogue, backward of
activation and bias, layer normalisation, 8-bit checkpoints, and the weight gradient from checkpoints.

Tolerances are elementwise bounds from the arithmetic, u = 2^-24 being half a step of fp32 and h half a step of the storage type:
  * one rounding to the storage type: h |value| (and the type's least step, for fp16's subnormals);
  * a sum of n products in fp32, in any order: n u sum |products|;
  * activations: a handful of fp32 operations and an exponential whose argument v carries an error of |v| u, |v| <= 16 where the
    step is not yet flat: 2^-19 of max(1, |z|) for the value, 2^-19 for the slope.
Every output lies between two strips of a marker value that have to survive, and starts as that marker itself."""
import math

import numpy as np
import pytest
import torch

import paper_2507_01154_amd as F
from oracle import flashdp_oracle as O
from gpu_util import DEV, env

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "fp32": torch.float32}
CODE = {"bf16": F.BF16, "f16": F.F16, "fp32": F.F32}
TINY = {"bf16": 2.0 ** -133, "f16": 2.0 ** -24, "fp32": 2.0 ** -149}
U = 2.0 ** -24
GUARD = 64
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


def half_step(dtype):
    return torch.finfo(TORCH[dtype]).eps / 2


class Out:
    """A device buffer of the given shape between two strips of a marker."""

    def __init__(self, shape, dtype):
        self.n = int(np.prod(shape))
        self.mark = 77 if dtype == torch.uint8 else 77.0
        self.all = torch.full((self.n + 2 * GUARD,), self.mark, dtype=dtype, device=DEV)
        self.t = self.all[GUARD:GUARD + self.n].view(shape)

    def cpu(self):
        torch.cuda.synchronize()
        assert bool((self.all[:GUARD] == self.mark).all()) and bool((self.all[GUARD + self.n:] == self.mark).all()), "written outside the output"
        return self.t.cpu().double() if self.t.dtype != torch.uint8 else self.t.cpu()


def rand(seed, shape, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(TORCH[dtype])


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "gelu":
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def quantise(x, f16):
    """(bytes as the buffer holds them, values) of rows in 8 bits; what is not finite is -128 and NaN."""
    x = x.double().numpy()
    rows, d = x.shape
    nb = -(-d // 32)
    p = np.zeros((rows, nb * 32))
    p[:, :d] = x
    p = p.reshape(rows, nb, 32)
    fin = np.isfinite(p)
    m = np.where(fin, np.abs(p), 0).max(-1)
    e = np.maximum(np.where(m > 0, np.frexp(np.where(m > 0, m, 1.0))[1] - 7, -999), -24 if f16 else -126)
    q = np.where(fin, np.clip(np.rint(np.ldexp(np.where(fin, p, 0), -e[..., None])), -127, 127), -128)
    v = np.where(fin, np.ldexp(q, e[..., None]), np.nan).reshape(rows, -1)[:, :d]
    qb = q.reshape(rows, -1)[:, :d].astype(np.int8).reshape(-1).view(np.uint8)
    return qb, (e + 127).astype(np.uint8).reshape(-1), torch.from_numpy(v.copy())


def packed_buffer(x, f16):
    qb, sb, v = quantise(x, f16)
    rows, d = x.shape
    buf = np.full(F.flashdp_checkpoint8_bytes(rows, d), 99, np.uint8)
    buf[:rows * d] = qb
    buf[len(buf) - len(sb):] = sb
    return torch.from_numpy(buf).to(DEV), v


def within(got, want, allowed, what=""):
    bad = (got - want).abs() > allowed
    assert not bool(bad.any()) and not bool(torch.isnan(got).any()), (
        what, int(bad.sum()), float(((got - want).abs() / allowed.clamp(min=1e-300)).max()))


# ---- forward product -------------------------------------------------------------------------------

FORWARD_SIZES = [(1, 1, 1), (1, 8, 8), (1, 768, 768), (2, 24, 40), (3, 7, 5), (5, 33, 31), (16, 64, 32), (17, 100, 65), (33, 129, 257), (64, 8, 1),
                 (1, 4096, 100), (7, 1000, 1003), (63, 72, 96), (65, 64, 64), (130, 200, 136), (257, 40, 264), (300, 520, 776), (1, 40, 2049), (48, 2056, 24)]


def run_forward(x, w, b, r, act, dtype, keep=None, inplace=False):
    rows, K = x.shape
    D = w.shape[0]
    y = Out((rows, D), TORCH[dtype])
    res = None
    if r is not None:
        res = r.to(DEV)
        if inplace:
            y.t.copy_(res)
            res = y.t
    z = None if keep is None else Out((F.flashdp_checkpoint8_bytes(rows, D),), torch.uint8) if keep == "8bit" else Out((rows, D), TORCH[dtype])
    F.flashdp_linear_forward(x.to(DEV), w.to(DEV), None if b is None else b.to(DEV), res, rows, K, D, CODE[dtype], act, y.t, None if z is None else z.t, keep == "8bit")
    return y.cpu(), None if z is None else z.cpu()


def check_forward(rows, K, D, dtype, act, bias, residual, keep, seed=0, inplace=False):
    x, w = rand(seed, (rows, K), dtype), rand(seed + 1, (D, K), dtype, max(K, 1) ** -0.5)
    b = rand(seed + 2, (D,), dtype) if bias else None
    r = rand(seed + 3, (rows, D), dtype) if residual else None
    y, z = run_forward(x, w, b, r, act, dtype, keep, inplace)
    x64, w64 = x.double(), w.double()
    z64 = x64 @ w64.T + (0 if b is None else b.double())
    slack = (K + 2) * U * (x64.abs() @ w64.abs().T + (0 if b is None else b.double().abs()))
    a64 = act64(z64, act)[0]
    y64 = a64 + (0 if r is None else r.double())
    h, tiny = half_step(dtype), TINY[dtype]
    act_err = torch.zeros_like(z64) if act in ("none", "relu") else 2.0 ** -19 * z64.abs().clamp(min=1)
    within(y, y64, (1 + h) * (1.13 * slack + act_err + 2 * U * y64.abs()) + h * y64.abs() + tiny, "y")
    if keep == "dtype":
        within(z, z64, (1 + h) * slack + h * z64.abs() + tiny, "z")
    elif keep == "8bit":
        back = Out((rows, D), TORCH[dtype])
        F.flashdp_checkpoint8_unpack(z.to(DEV), rows, D, CODE[dtype], back.t)
        nb = -(-D // 32)
        m = torch.nn.functional.pad((z64.abs() + slack), (0, nb * 32 - D)).view(rows, nb, 32).amax(-1).repeat_interleave(32, 1)[:, :D]
        within(back.cpu(), z64, m / 64 + slack + tiny, "z in 8 bits")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
@pytest.mark.parametrize("rows,K,D", FORWARD_SIZES)
def test_forward_sizes(rows, K, D, dtype):
    check_forward(rows, K, D, dtype, "none", False, False, None)
    check_forward(rows, K, D, dtype, "silu", True, True, "dtype", seed=5)
    check_forward(rows, K, D, dtype, "gelu_tanh", True, False, "8bit", seed=9)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows", [1, 20, 200])
def test_forward_epilogues(rows, act, dtype):
    for k, (bias, residual, keep) in enumerate([(False, True, None), (True, False, "dtype"), (True, True, "8bit"), (False, False, "8bit")]):
        check_forward(rows, 136, 200, dtype, act, bias, residual, keep, seed=20 + k)
    check_forward(rows, 136, 200, dtype, act, True, True, None, seed=30, inplace=True)      # added to the residual in place


# the kernels of the ladder (0 to 6: rows of whole 16-byte chunks; 4 and 6 are not made for fp32), those for other rows (7 to 9) and those of fp32
# in bfloat16 parts (10, 11), on sizes that leave them ragged edges, one k-tile and many, and more k-tiles than stages
FORCED = [(k, r, K, D) for k in range(7) for r, K, D in [(1, 8, 8), (5, 64, 40), (33, 136, 72), (70, 1160, 136), (300, 520, 328)]] + \
         [(k, r, K, D) for k in (7, 8, 9) for r, K, D in [(1, 1, 8), (5, 63, 40), (33, 137, 75), (64, 1161, 137), (150, 517, 329)]] + \
         [(k, r, K, D) for k in (10, 11) for r, K, D in [(1, 64, 8), (70, 1161, 137), (300, 520, 328), (150, 66, 600)]]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
@pytest.mark.parametrize("kernel,rows,K,D", FORCED)
def test_every_forward_kernel(kernel, rows, K, D, dtype):
    with env(FLASHDP_FORWARD=kernel):
        check_forward(rows, K, D, dtype, "none", False, False, None, seed=40)
        check_forward(rows, K, D, dtype, "gelu", True, True, "dtype", seed=50)
        check_forward(rows, K, D, dtype, "silu", True, False, "8bit", seed=60)
        want = {7: "forward_rows_kernel" if rows <= 64 else "forward_tile_kernel", 8: "forward_tile_kernel", 9: "forward_tile_kernel",
                5: "forward_large_kernel", 6: "forward_large_kernel", 10: "forward_split_kernel", 11: "forward_split_kernel"}.get(kernel, "forward_deep_kernel")
        if (kernel < 10 and dtype != "fp32") or (kernel not in (4, 6) and dtype == "fp32"):
            assert F.flashdp_last_kernel() == want or kernel == 0           # (8-bit blocks of 32 features are wider than the smallest tile)


@pytest.mark.parametrize("rows,K,D,dtype", [(1024, 768, 2304, "bf16"), (777, 1096, 2312, "f16"), (520, 1001, 1003, "bf16"), (512, 768, 776, "fp32"), (1500, 515, 770, "fp32"),
                                            (4096, 256, 4096, "bf16"), (4099, 264, 4104, "f16"), (2100, 192, 8208, "fp32"), (2, 13824, 5120, "bf16"), (8, 768, 50257, "f16")])
def test_forward_large(rows, K, D, dtype):
    """Against float64 on the device's own matrix product (its error is of another order than the bound)."""
    x, w = rand(1, (rows, K), dtype).to(DEV), rand(2, (D, K), dtype, K ** -0.5).to(DEV)
    b, r = rand(3, (D,), dtype).to(DEV), rand(4, (rows, D), dtype).to(DEV)
    y, z = Out((rows, D), TORCH[dtype]), Out((rows, D), TORCH[dtype])
    F.flashdp_linear_forward(x, w, b, r, rows, K, D, CODE[dtype], "gelu_tanh", y.t, z.t)
    z64 = x.double() @ w.double().T + b.double()
    slack = (K + 2) * U * (x.double().abs() @ w.double().abs().T + b.double().abs())
    y64 = act64(z64, "gelu_tanh")[0] + r.double()
    h, tiny = half_step(dtype), TINY[dtype]
    yc, zc = y.cpu().to(DEV), z.cpu().to(DEV)
    within(zc, z64, (1 + h) * slack + h * z64.abs() + tiny, "z")
    within(yc, y64, (1 + h) * (1.13 * slack + 2.0 ** -19 * z64.abs().clamp(min=1) + 2 * U * y64.abs()) + h * y64.abs() + tiny, "y")
    # bounds of the worst case are loose by sqrt(K): the error in norm is that of one rounding, fp32 sums beside it
    assert float((yc - y64).norm() / y64.norm()) <= h + 2 * math.sqrt(K) * U


@pytest.mark.parametrize("kernel", [10, 11])
def test_parts_of_floats_over_the_range_of_their_exponents(kernel):
    """fp32 in bfloat16 parts: rows of X scaled from 2^-100 to 2^100 (down to where the third part is a normal number), values with all 24 bits
    set, powers of two, the largest number, and rows that are not finite, which spoil themselves alone."""
    rows, K, D = 40, 136, 72
    x, w = rand(1, (rows, K), "fp32"), rand(2, (D, K), "fp32")
    x *= torch.logspace(-100, 100, rows, base=2)[:, None]
    x[3], x[4] = float(2 ** 24 - 1), 2.0 ** torch.arange(-60, 76).float()
    x[5] = 0.0
    x[5, 0] = torch.finfo(torch.float32).max
    x[6, 1], x[7, 2] = math.nan, math.inf
    with env(FLASHDP_FORWARD=kernel):
        y, _ = run_forward(x, w * 0.5, None, None, None, "fp32")
        assert F.flashdp_last_kernel() == "forward_split_kernel"
    x64, w64 = x.double(), w.double() * 0.5
    fine = torch.ones(rows, dtype=torch.bool)
    fine[6:8] = False
    y64, mag = (x64 @ w64.T)[fine], (x64[fine].abs() @ w64.abs().T)
    assert not torch.isfinite(y[~fine]).any()
    got = y[fine]
    over = y64.abs() > 3.4e38
    within(got[~over], y64[~over], ((K + 2) * U * mag + 1e-45)[~over])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
def test_forward_values_that_are_not_finite_stay_in_their_row_and_column(dtype):
    rows, K, D = 70, 72, 100
    x, w, b = rand(1, (rows, K), dtype), rand(2, (D, K), dtype), rand(3, (D,), dtype)
    clean, _ = run_forward(x, w, b, None, "silu", dtype)
    x[5, 3], x[69, 71] = math.nan, math.inf
    w[7, 0] = math.nan
    b[11] = -math.inf
    got, z8 = run_forward(x, w, b, None, "silu", dtype, "8bit")
    touched = torch.zeros(rows, D, dtype=torch.bool)
    touched[5], touched[69], touched[:, 7] = True, True, True
    assert torch.isnan(got[5]).all() and torch.isnan(got[:, 7]).all()
    touched[:, 11] = True
    assert bool((got[:, 11][torch.arange(rows) != 5][:-1] == 0).all())      # the limit of silu, not infinity times zero
    assert torch.equal(got[~touched], clean[~touched])
    back = Out((rows, D), TORCH[dtype])
    F.flashdp_checkpoint8_unpack(z8.to(DEV), rows, D, CODE[dtype], back.t)
    back = back.cpu()
    assert torch.isnan(back[touched]).all() and not torch.isnan(back[~touched]).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_activations_reach_their_limits(dtype):
    """One feature, W = 1: Z is the input itself, over the whole range of the type."""
    v = torch.tensor([-math.inf, -3e38, -1e20, -200.0, -30.0, -1.0, -0.0, 0.0, 1e-30, 0.5, 30.0, 200.0, 1e20, 3e38, math.inf, math.nan]).to(TORCH[dtype])
    for act in ACTS[1:]:
        y, _ = run_forward(v[:, None].contiguous(), torch.ones(1, 1, dtype=TORCH[dtype]), None, None, act, dtype)
        y = y[:, 0]
        assert bool((y[:4].abs() <= 1e-30).all()) and torch.isnan(y[-1]) and y[-2] == math.inf
        assert torch.equal(y[11:14], v[11:14].double())
        dz, g = Out((16, 1, 1), TORCH[dtype]), Out((1,), torch.float32)
        F.flashdp_activation_dp_grad(torch.ones(16, 1, 1, dtype=TORCH[dtype], device=DEV), v.to(DEV), False, 16, 1, 1, CODE[dtype], act, 1.0, 0.0, 0, 0, dz.t, None)
        s = dz.cpu().reshape(-1)
        assert bool((s[:4].abs() <= 1e-30).all()) and bool((s[11:15] == 1).all()) and torch.isnan(s[-1])
        assert bool(s[7] == (0.0 if act == "relu" else 0.5))


# ---- activation and bias ---------------------------------------------------------------------------

def clipped64(G, C, sigma, seed, layer, field):
    """The oracle's stages 2 to 4 on per-sample vectors G [B, n]; the noise of a vector's own field."""
    norms = G.square().sum(1).sqrt()
    c = torch.tensor([O.clip_factor(float(n), C) for n in norms])
    out = (c[:, None] * G).sum(0)
    if sigma:
        n = out.numel()
        groups = np.arange((n + 3) // 4, dtype=np.uint64)
        ctr = np.zeros((groups.size, 4), np.uint32)
        ctr[:, 0], ctr[:, 1], ctr[:, 2], ctr[:, 3] = groups & np.uint64(0xFFFFFFFF), groups >> np.uint64(32), layer, field
        z = O.gaussians_from_words(O.philox4x32_10(ctr, (seed & 0xFFFFFFFF, seed >> 32))).reshape(-1)[:n]
        out = out + sigma * C * torch.from_numpy(z.copy())
    return out, norms, c


def check_vector(g, n, G, err, C, sigma, seed, layer, field):
    """out_grad and norms of per-sample vectors G whose elements carry errors up to err [B, n]."""
    want, norms, c = clipped64(G, C, sigma, seed, layer, field)
    dn = err.square().sum(1).sqrt()
    within(n, norms, dn + 4 * U * norms + 1e-37, "norms")
    rel = dn / norms.clamp(min=1e-300)
    B = G.shape[0]
    allowed = (c[:, None] * (err + (rel[:, None] + (B + 4) * U) * G.abs())).sum(0) + sigma * C * 2e-6 + 4 * U * want.abs() + 1e-37
    within(g, want, allowed, "gradient")


VECTOR_SIZES = [(1, 1, 1), (1, 1, 8), (2, 1, 40), (300, 1, 7), (1, 5, 33), (3, 4, 64), (2, 17, 100), (5, 33, 513), (1, 300, 72), (4, 129, 1001), (2, 64, 2056), (70, 3, 24), (1, 1, 5003)]


def check_activation(B, T, d, dtype, act, keep, C, sigma, inplace=False):
    scale = torch.tensor([10.0 ** ((i % 5) - 2) for i in range(B)])[:, None, None]
    dy = (rand(1, (B, T, d), "fp32") * scale).to(TORCH[dtype])
    z = rand(2, (B * T, d), dtype, 2.0)
    zdev = None
    if keep == "8bit":
        zdev, z64 = packed_buffer(z, dtype == "f16")
    else:
        z64 = z.double()
        zdev = z.to(DEV) if act != "none" else None
    dz, g, n = Out((B, T, d), TORCH[dtype]), Out((d,), torch.float32), Out((B,), torch.float32)
    dydev = dy.to(DEV)
    if inplace:
        dz.t.copy_(dydev)
        dydev = dz.t
    F.flashdp_activation_dp_grad(dydev, zdev, keep == "8bit", B, T, d, CODE[dtype], act, C, sigma, 5 + (9 << 32), 3, dz.t if act != "none" or inplace else None, g.t, n.t)
    dy64 = dy.double()
    slope = act64(z64, act)[1].view(B, T, d)
    dz64 = dy64 * slope
    serr = torch.zeros_like(dz64) if act in ("none", "relu") else 2.0 ** -19 * dy64.abs()
    h = half_step(dtype)
    if act != "none" or inplace:
        within(dz.cpu(), dz64, (1 + h) * (serr + 2 * U * dz64.abs()) + h * dz64.abs() + TINY[dtype], "dz")
    err = serr.sum(1) + (T + 2) * U * dz64.abs().sum(1)
    check_vector(g.cpu(), n.cpu(), dz64.sum(1), err, C, sigma, 5 + (9 << 32), 3, F.FIELD_BIAS)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
@pytest.mark.parametrize("B,T,d", VECTOR_SIZES)
def test_activation_sizes(B, T, d, dtype):
    check_activation(B, T, d, dtype, "gelu_tanh", "8bit", 1.0, 0.0)
    check_activation(B, T, d, dtype, "silu", "dtype", 0.5, 0.7)
    check_activation(B, T, d, dtype, "none", "none", 2.0, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("act", ACTS[1:])
@pytest.mark.parametrize("T", [1, 50])
def test_activation_kinds(act, T, dtype):
    for keep in ("dtype", "8bit"):
        check_activation(6, T, 200, dtype, act, keep, 1.0, 0.3)
    check_activation(6, T, 203, dtype, act, "dtype", 1e6, 0.0, inplace=True)        # nothing clips; dZ over dY


def test_activation_without_a_bias_and_bias_without_an_activation():
    dy, z = rand(1, (3, 20, 72), "bf16").to(DEV), rand(2, (60, 72), "bf16").to(DEV)
    full, dz = Out((3, 20, 72), torch.bfloat16), Out((3, 20, 72), torch.bfloat16)
    g, n = Out((72,), torch.float32), Out((3,), torch.float32)
    F.flashdp_activation_dp_grad(dy, z, False, 3, 20, 72, F.BF16, "gelu", 1.0, 0.0, 0, 0, full.t, g.t, n.t)
    F.flashdp_activation_dp_grad(dy, z, False, 3, 20, 72, F.BF16, "gelu", 0.0, -1.0, 0, 0, dz.t, None)         # C, sigma unused
    assert torch.equal(full.cpu(), dz.cpu())
    g2, n2 = Out((72,), torch.float32), Out((3,), torch.float32)
    F.flashdp_activation_dp_grad(dy, z, False, 3, 20, 72, F.BF16, "gelu", 1.0, 0.0, 0, 0, None, g2.t, n2.t)
    assert torch.equal(g.cpu(), g2.cpu()) and torch.equal(n.cpu(), n2.cpu())


def test_vector_gradients_accumulate_over_micro_batches_with_noise_once():
    B, T, d = 6, 9, 136
    dy = rand(1, (B, T, d), "fp32", 3.0)
    g, n = Out((d,), torch.float32), Out((B,), torch.float32)
    for k, (a, b) in enumerate([(0, 1), (1, 4), (4, 6)]):
        F.flashdp_activation_dp_grad(dy[a:b].to(DEV), None, False, b - a, T, d, F.F32, None, 2.0, 0.5, 7, 1, None, g.t, n.t[a:b], accumulate=k > 0, add_noise=k == 2)
    err = (T + 2) * U * dy.double().abs().sum(1)
    check_vector(g.cpu(), n.cpu(), dy.double().sum(1), err, 2.0, 0.5, 7, 1, F.FIELD_BIAS)


@pytest.mark.parametrize("B,blocks", [(1030, 1), (1023, 9)])
def test_more_samples_than_a_workgroup_holds_factors_of(B, blocks):
    d = 64 * blocks - 3
    dy = rand(4, (B, 1, d), "fp32") * torch.logspace(-2, 2, B)[:, None, None]
    g, n = Out((d,), torch.float32), Out((B,), torch.float32)
    F.flashdp_activation_dp_grad(dy.to(DEV), None, False, B, 1, d, F.F32, None, 1.0, 0.0, 7, 1, None, g.t, n.t)
    check_vector(g.cpu(), n.cpu(), dy[:, 0].double(), 2 * U * dy[:, 0].double().abs(), 1.0, 0.0, 7, 1, F.FIELD_BIAS)


def test_norms_that_overflow_fp32_squares_are_norms_and_nan_poisons():
    dy = torch.ones(3, 2, 40)
    dy[0] *= 1e25
    g, n = Out((40,), torch.float32), Out((3,), torch.float32)
    call = lambda: F.flashdp_activation_dp_grad(dy.to(DEV), None, False, 3, 2, 40, F.F32, None, 1.0, 0.0, 7, 1, None, g.t, n.t)   # noqa: E731
    call()
    check_vector(g.cpu(), n.cpu(), dy.double().sum(1), 8 * U * dy.double().sum(1), 1.0, 0.0, 7, 1, F.FIELD_BIAS)
    dy[1, 0, 5] = math.nan
    call()
    assert torch.isnan(g.cpu()).all() and torch.isnan(n.cpu()[1]) and not torch.isnan(n.cpu()[2])


# ---- layer normalisation ---------------------------------------------------------------------------

NORM_SIZES = [(1, 1, 1), (1, 1, 2), (1, 1, 8), (2, 1, 33), (1, 7, 64), (3, 5, 100), (2, 33, 768), (5, 3, 1000), (1, 1, 5120), (2, 9, 1025), (1, 20, 2056), (2, 3, 4104), (1, 5, 6152),
              (300, 1, 24), (2, 2, 8200), (1, 3, 16400), (2, 2, 20001), (1, 40, 515)]


def check_norm(B, T, d, dtype, bias=True, C=1.0, sigma=0.0, offset=0.5, inplace=False, eps=1e-5):
    rows = B * T
    x = (rand(1, (rows, d), "fp32") * torch.linspace(0.1, 3, d) + offset).to(TORCH[dtype])
    w = (1 + 0.2 * rand(2, (d,), "fp32")).to(TORCH[dtype])
    b = rand(3, (d,), dtype) if bias else None
    scale = torch.tensor([10.0 ** ((i % 4) - 2) for i in range(B)])[:, None, None]
    dy = (rand(4, (B, T, d), "fp32") * scale).to(TORCH[dtype])
    f = TORCH[dtype]
    y, mean, rstd = Out((rows, d), f), Out((rows,), torch.float32), Out((rows,), torch.float32)
    xd, wd = x.to(DEV), w.to(DEV)
    F.flashdp_layernorm_forward(xd, wd, None if b is None else b.to(DEV), rows, d, CODE[dtype], eps, y.t, mean.t, rstd.t)
    dx, g, n = Out((B, T, d), f), Out((2 if bias else 1, d), torch.float32), Out((B,), torch.float32)
    dyd = dy.to(DEV)
    if inplace:
        dx.t.copy_(dyd)
        dyd = dx.t
    F.flashdp_layernorm_dp_grad(xd, dyd, wd, mean.t, rstd.t, B, T, d, CODE[dtype], C, sigma, 11, 2, dx.t, g.t, n.t, bias)
    x64, w64, dy64 = x.double(), w.double(), dy.double().view(rows, d)
    mu = x64.mean(1, keepdim=True)
    var = (x64 - mu).square().mean(1, keepdim=True)
    r = (var + eps) ** -0.5
    xh = (x64 - mu) * r
    h, tiny = half_step(dtype), TINY[dtype]
    # sums of a row: up to d / 64 + 10 additions one after the other
    k = (d / 64 + 10) * U
    emu = k * x64.abs().mean(1, keepdim=True) + U * mu.abs()
    er = (k + 4 * U) + (emu * r) ** 2        # relative error of rstd: half that of the variance, into which the mean's error goes squared
    within(mean.cpu(), mu[:, 0], emu[:, 0] + 1e-38, "mean")
    within(rstd.cpu(), r[:, 0], er[:, 0] * r[:, 0], "rstd")
    exh = emu * r + (er + 3 * U) * xh.abs()
    b64 = 0 if b is None else b.double()
    y64 = xh * w64 + b64
    within(y.cpu(), y64, (1 + h) * (exh * w64.abs() + 3 * U * (xh * w64).abs() + 2 * U * y64.abs()) + h * y64.abs() + tiny, "y")
    a = dy64 * w64
    m0, m1 = a.mean(1, keepdim=True), (a * xh).mean(1, keepdim=True)
    em0 = (k + 3 * U) * a.abs().mean(1, keepdim=True)
    em1 = (k + 3 * U) * (a * xh).abs().mean(1, keepdim=True) + (a.abs() * exh).mean(1, keepdim=True)
    dx64 = r * (a - m0 - xh * m1)
    edx = r * (4 * U * a.abs() + em0 + xh.abs() * em1 + exh * m1.abs() + 4 * U * (a.abs() + m0.abs() + (xh * m1).abs())) + er * dx64.abs()
    within(dx.cpu().view(rows, d), dx64, (1 + h) * edx + h * dx64.abs() + tiny, "dx")
    per = lambda t: t.view(B, T, d).sum(1)     # noqa: E731
    gw, ew = per(dy64 * xh), per(dy64.abs() * exh) + (T + 3) * U * per((dy64 * xh).abs())
    G, err = (torch.cat((gw, per(dy64)), 1), torch.cat((ew, (T + 3) * U * per(dy64.abs())), 1)) if bias else (gw, ew)
    check_vector(g.cpu().reshape(-1), n.cpu(), G, err, C, sigma, 11, 2, F.FIELD_NORM)
    if inplace:      # Y over X, too
        over = Out((rows, d), f)
        over.t.copy_(xd)
        F.flashdp_layernorm_forward(over.t, wd, None if b is None else b.to(DEV), rows, d, CODE[dtype], eps, over.t)
        assert torch.equal(over.cpu(), y.cpu())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
@pytest.mark.parametrize("B,T,d", NORM_SIZES)
def test_layernorm_sizes(B, T, d, dtype):
    check_norm(B, T, d, dtype)
    check_norm(B, T, d, dtype, bias=False, sigma=0.6, inplace=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [96, 1032, 20000])
def test_layernorm_of_a_stream_with_a_large_offset(d, dtype):
    """Mean 300 and deviations of about one: a mean of squares minus a squared mean would have lost five digits."""
    check_norm(2, 4, d, dtype, offset=300.0)


@pytest.mark.parametrize("d", [40, 1500, 17000])
def test_constant_rows_and_rows_that_are_not_finite(d):
    x = torch.full((4, d), 3.0)
    x[1] = rand(1, (d,), "fp32")
    x[2] = rand(2, (d,), "fp32")
    x[2, d // 2] = math.nan
    y, mean, rstd = Out((4, d), torch.float32), Out((4,), torch.float32), Out((4,), torch.float32)
    w, b = torch.full((d,), 2.0, device=DEV), torch.full((d,), 0.25, device=DEV)
    F.flashdp_layernorm_forward(x.to(DEV), w, b, 4, d, F.F32, 1e-5, y.t, mean.t, rstd.t)
    yc = y.cpu()
    assert bool((yc[0] == 0.25).all()) and bool((yc[3] == 0.25).all()) and torch.isnan(yc[2]).all() and not torch.isnan(yc[1]).any()
    assert abs(float(rstd.cpu()[0]) - 1e-5 ** -0.5) <= 1e-4
    only = Out((4, d), torch.float32)
    F.flashdp_layernorm_forward(x.to(DEV), w, b, 4, d, F.F32, 1e-5, only.t)                 # inference: nothing kept
    assert torch.equal(only.cpu()[:2], yc[:2])


def test_layernorm_gradients_agree_with_differences():
    """d<dY, Y>/dx and d<dY, Y>/dgamma by central differences in 64 bits of the definition, against the kernels."""
    d, eps = 24, 1e-5
    x, w, b, dy = rand(1, (1, d), "fp32"), 1 + rand(2, (d,), "fp32", 0.1), rand(3, (d,), "fp32"), rand(4, (1, 1, d), "fp32")
    f = lambda x, w, b: float((dy.double()[0] * ((x - x.mean()) * (((x - x.mean()) ** 2).mean() + eps) ** -0.5 * w + b)).sum())   # noqa: E731
    y, mean, rstd = Out((1, d), torch.float32), Out((1,), torch.float32), Out((1,), torch.float32)
    F.flashdp_layernorm_forward(x.to(DEV), w.to(DEV), b.to(DEV), 1, d, F.F32, eps, y.t, mean.t, rstd.t)
    dx, g = Out((1, 1, d), torch.float32), Out((2, d), torch.float32)
    F.flashdp_layernorm_dp_grad(x.to(DEV), dy.to(DEV), w.to(DEV), mean.t, rstd.t, 1, 1, d, F.F32, 1e6, 0.0, 0, 0, dx.t, g.t)
    at = [x.double()[0], w.double(), b.double()]
    step = 1e-5
    for k, got in enumerate((dx.cpu().reshape(-1), g.cpu()[0], g.cpu()[1])):
        for e in range(d):
            lo, hi = [t.clone() for t in at], [t.clone() for t in at]
            lo[k][e] -= step
            hi[k][e] += step
            assert abs((f(*hi) - f(*lo)) / (2 * step) - float(got[e])) <= 2e-5 * (1 + abs(float(got[e])))


# ---- 8-bit checkpoints -----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 31), (1, 32), (3, 33), (2, 40), (7, 64), (5, 100), (64, 768), (33, 1001), (1, 5120), (129, 24)])
def test_checkpoint_bytes_and_values(rows, d, dtype):
    x = rand(rows + d, (rows, d), dtype) * 2.0 ** torch.randint(-20, 12, (rows, 1), generator=torch.Generator().manual_seed(d)).to(TORCH[dtype])
    if d > 40:
        x[0, :32] = 0
    qb, sb, v = quantise(x, dtype == "f16")
    p = Out((F.flashdp_checkpoint8_bytes(rows, d),), torch.uint8)
    F.flashdp_checkpoint8_pack(x.to(DEV), rows, d, CODE[dtype], p.t)
    got = p.cpu().numpy()
    assert np.array_equal(got[:rows * d], qb) and np.array_equal(got[got.size - sb.size:], sb)
    assert bool((p.t[rows * d:p.n - sb.size] == p.mark).all())                      # the padding is not written
    y = Out((rows, d), TORCH[dtype])
    F.flashdp_checkpoint8_unpack(p.t, rows, d, CODE[dtype], y.t)
    assert torch.equal(y.cpu(), v)
    # and what came back packs to the same values: nothing moves the second time
    p2, y2 = Out((p.n,), torch.uint8), Out((rows, d), TORCH[dtype])
    F.flashdp_checkpoint8_pack(y.t, rows, d, CODE[dtype], p2.t)
    F.flashdp_checkpoint8_unpack(p2.t, rows, d, CODE[dtype], y2.t)
    assert torch.equal(y2.cpu(), v)
    m = torch.nn.functional.pad(x.double().abs(), (0, -d % 32)).view(rows, -1, 32).amax(-1).repeat_interleave(32, 1)[:, :d]
    assert bool(((v - x.double()).abs() <= m / 64).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
def test_checkpoint_of_extreme_values(dtype):
    """Blocks of the type's largest and smallest values, of zeros, ties, and of values that are not finite."""
    fi = torch.finfo(TORCH[dtype])
    x = torch.zeros(8, 32, dtype=TORCH[dtype])
    x[0, :4] = torch.tensor([fi.max, -fi.max, fi.max / 2, 1.0]).to(TORCH[dtype])
    x[1, :3] = torch.tensor([fi.tiny, -fi.tiny, fi.tiny / 2]).to(TORCH[dtype])
    x[2, :2] = torch.tensor([TINY[dtype], -3 * TINY[dtype]]).to(TORCH[dtype])
    x[4, :6] = torch.tensor([64.0, 0.5, 1.5, 2.5, -0.5, -3.5]).to(TORCH[dtype])      # step 1: ties to even
    x[5, :3] = torch.tensor([127.5, -127.5, 1.0]).to(TORCH[dtype])                   # cut to 127
    x[6, :4] = torch.tensor([math.nan, math.inf, -math.inf, 5.0]).to(TORCH[dtype])
    x[7] = math.nan
    qb, sb, v = quantise(x, dtype == "f16")
    p, y = Out((F.flashdp_checkpoint8_bytes(8, 32),), torch.uint8), Out((8, 32), TORCH[dtype])
    F.flashdp_checkpoint8_pack(x.to(DEV), 8, 32, CODE[dtype], p.t)
    F.flashdp_checkpoint8_unpack(p.t, 8, 32, CODE[dtype], y.t)
    got = p.cpu().numpy()
    assert np.array_equal(got[:256], qb) and np.array_equal(got[256:], sb)
    yc = y.cpu()
    assert torch.equal(torch.isnan(yc), torch.isnan(v)) and torch.equal(torch.nan_to_num(yc), torch.nan_to_num(v))
    assert list(yc[4, :6]) == [64, 0, 2, 2, 0, -4] and list(yc[5, :2]) == [127, -127]


# ---- weight gradients from checkpoints -------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp32"])
@pytest.mark.parametrize("schedule", ["auto", "twopass", "scratch"])
@pytest.mark.parametrize("B,T,P,D", [(1, 1, 8, 8), (3, 1, 40, 24), (4, 16, 32, 32), (2, 40, 100, 33), (3, 200, 264, 136), (2, 33, 31, 65)])
def test_gradient_from_checkpoints_is_the_gradient_at_the_kept_values(B, T, P, D, schedule, dtype):
    x, dy = rand(1, (B * T, P), dtype), rand(2, (B, T, D), dtype)
    buf, v = packed_buffer(x, dtype == "f16")
    out, n = Out((D, P), torch.float32), Out((B,), torch.float32)
    L = [dict(X=buf, dY=dy.to(DEV), d_in=P, d_out=D, C=1.5, sigma=0.5, seed=3, layer=4, out_grad=out.t, out_norms=n.t)]
    F.flashdp_block_dp_grad_checkpoint8(L, B, T, CODE[dtype], schedule)
    want, wn = Out((D, P), torch.float32), Out((B,), torch.float32)
    ws = torch.empty((max(F.flashdp_workspace_bytes([dict(L[0], X=None)], B, T, CODE[dtype], schedule), 16),), dtype=torch.uint8, device=DEV)
    F.flashdp_block_dp_grad([dict(L[0], X=v.to(TORCH[dtype]).to(DEV), out_grad=want.t, out_norms=wn.t)], B, T, CODE[dtype], schedule, ws)
    assert torch.equal(out.cpu(), want.cpu()) and torch.equal(n.cpu(), wn.cpu())
    if schedule == "twopass":       # and that is the definition's
        x64, dy64 = v.view(B, T, P), dy.double()
        G = dy64.transpose(1, 2).contiguous() @ x64
        err = (T + 2) * U * (dy64.abs().transpose(1, 2).contiguous() @ x64.abs())
        w64, norms, c = clipped64(G.reshape(B, -1), 1.5, 0.0, 3, 4, 0)
        w64 = w64 + 0.75 * torch.from_numpy(O.noise_field(3, 4, D * P))
        e = err.reshape(B, -1)
        rel = e.square().sum(1).sqrt() / norms + 8 * U
        allowed = (c[:, None] * (e + (rel[:, None] + 4 * B * U) * G.reshape(B, -1).abs())).sum(0) + 0.75 * 2e-6 + 4 * U * w64.abs()
        within(out.cpu().reshape(-1), w64, allowed)


def test_layers_that_share_a_checkpoint_and_micro_batches():
    """Three layers on one activation and one on another, in two micro-batches: each as by itself."""
    B, T, P, D = 4, 24, 72, 40
    code = F.BF16
    x = [rand(k, (B * T, P), "bf16") for k in range(2)]
    bufs = [[packed_buffer(t.view(B, T, P)[h].reshape(-1, P), False)[0] for h in (slice(0, 2), slice(2, 4))] for t in x]
    dy = [rand(10 + k, (B, T, D), "bf16") for k in range(4)]
    use = [0, 0, 0, 1]
    outs = [Out((D, P), torch.float32) for _ in use]
    alone = [Out((D, P), torch.float32) for _ in use]
    for h in range(2):
        part = slice(2 * h, 2 * h + 2)
        mk = lambda k, o: dict(X=bufs[use[k]][h], dY=dy[k][part].contiguous().to(DEV), d_in=P, d_out=D, C=1.0 + k, sigma=0.5, seed=3, layer=k, out_grad=o.t, out_norms=None)   # noqa: E731
        F.flashdp_block_dp_grad_checkpoint8([mk(k, outs[k]) for k in range(4)], 2, T, code, "twopass", accumulate=h > 0, add_noise=h == 1)
        for k in range(4):
            F.flashdp_block_dp_grad_checkpoint8([mk(k, alone[k])], 2, T, code, "twopass", accumulate=h > 0, add_noise=h == 1)
    for a, b in zip(outs, alone):
        a, b = a.cpu(), b.cpu()
        assert float((a - b).norm() / b.norm()) <= 1e-6


# ---- streams, workspaces, graphs, repetition -------------------------------------------------------

def everything(dtype="bf16", B=3, T=70, P=200, D=136):
    """All calls once, in the order of a layer's forward and backward pass, on buffers of their own; returns (call, outputs)."""
    f, code, rows = TORCH[dtype], CODE[dtype], B * T
    new = lambda *s, dtype=f: torch.empty(s, dtype=dtype, device=DEV)      # noqa: E731
    x, w, b = rand(1, (rows, P), dtype).to(DEV), rand(2, (D, P), dtype, P ** -0.5).to(DEV), rand(3, (D,), dtype).to(DEV)
    gam, bet = rand(4, (P,), dtype).to(DEV), rand(5, (P,), dtype).to(DEV)
    dy = rand(6, (B, T, D), dtype).to(DEV)
    h, mean, rstd = new(rows, P), new(rows, dtype=torch.float32), new(rows, dtype=torch.float32)
    h8, z8 = (new(F.flashdp_checkpoint8_bytes(rows, n), dtype=torch.uint8) for n in (P, D))
    y, dz, dh, dx = new(rows, D), new(B, T, D), new(B, T, P), new(B, T, P)
    gb, gw, gn = new(D, dtype=torch.float32), new(D, P, dtype=torch.float32), new(2, P, dtype=torch.float32)
    nb, nw, nn = (new(B, dtype=torch.float32) for _ in range(3))
    L = F.make_layers([dict(X=h8, dY=dz, d_in=P, d_out=D, C=1.0, sigma=0.5, seed=1, layer=0, out_grad=gw, out_norms=nw)])
    room = lambda n: new(n, dtype=torch.uint8)     # noqa: E731
    wa, wn = room(F.flashdp_activation_workspace_bytes(B, T, D, code)), room(F.flashdp_layernorm_workspace_bytes(B, T, P, code))
    wg = room(F.flashdp_workspace_bytes_checkpoint8(L, B, T, code, "twopass"))

    def call():
        F.flashdp_layernorm_forward(x, gam, bet, rows, P, code, 1e-5, h, mean, rstd)
        F.flashdp_checkpoint8_pack(h, rows, P, code, h8)
        F.flashdp_linear_forward(h, w, b, None, rows, P, D, code, "gelu_tanh", y, z8, True)
        F.flashdp_activation_dp_grad(dy, z8, True, B, T, D, code, "gelu_tanh", 1.0, 0.5, 1, 0, dz, gb, nb, wa)
        F.flashdp_block_dp_grad_checkpoint8(L, B, T, code, "twopass", wg)
        torch.matmul(dz, w, out=dh)
        F.flashdp_layernorm_dp_grad(x, dh, gam, mean, rstd, B, T, P, code, 1.0, 0.5, 1, 0, dx, gn, nn, True, wn)

    return call, [h, mean, rstd, h8, z8, y, dz, gb, nb, gw, nw, dx, gn, nn], [wa, wn, wg]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_calls_repeat_to_the_bit_and_replay_from_a_graph(dtype):
    call, outs, rooms = everything(dtype)
    call()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for rep in range(4):
        for o in outs:
            o.fill_(99 if o.dtype == torch.uint8 else float("nan"))
        for r in rooms:
            r.random_(0, 255)              # eager work between replays; nothing may depend on what a workspace holds
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for o, v in zip(outs, want):
            if o.dtype != torch.uint8:     # (a checkpoint's padding is not written)
                assert torch.equal(o, v), rep


def test_two_graphs_with_workspaces_of_their_own_replay_in_turn():
    pairs = [everything("bf16", 3, 70, 200, 136), everything("bf16", 2, 33, 96, 264)]
    want, graphs = [], []
    for call, outs, _ in pairs:
        call()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for k in order:
            for o in pairs[k][1]:
                o.fill_(99 if o.dtype == torch.uint8 else float("nan"))
            graphs[k].replay()
        torch.cuda.synchronize()
        for k in (0, 1):
            assert all(torch.equal(o, v) for o, v in zip(pairs[k][1], want[k]) if o.dtype != torch.uint8)


def test_other_streams_side_by_side():
    """Two streams with buffers and workspaces of their own give what one after the other gives."""
    pairs = [everything("bf16", 3, 70, 200, 136), everything("fp32", 4, 31, 104, 72)]
    want = []
    for call, outs, _ in pairs:
        call()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
        for o in outs:
            o.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(3):
        for (call, _, _), s in zip(pairs, streams):
            with torch.cuda.stream(s):
                call()
    torch.cuda.synchronize()
    for (_, outs, _), w in zip(pairs, want):
        assert all(torch.equal(o, v) for o, v in zip(outs, w) if o.dtype != torch.uint8)


def test_the_library_workspace_is_not_grown_while_a_graph_is_captured():
    F.flashdp_release()
    dy, g = torch.zeros(2, 40, 64, device=DEV), torch.zeros(64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(F.FlashDPError) as e:
            F.flashdp_activation_dp_grad(dy, None, False, 2, 40, 64, F.F32, None, 1.0, 0.0, 0, 0, None, g)
        assert e.value.status == F.WORKSPACE_TOO_SMALL
        g.add_(1.0)                     # the capture goes on
    graph.replay()
    torch.cuda.synchronize()
    assert float(g.sum()) == 64.0
    F.flashdp_activation_dp_grad(dy, None, False, 2, 40, 64, F.F32, None, 1.0, 0.0, 0, 0, None, g)
    torch.cuda.synchronize()
    assert float(g.abs().sum()) == 0.0


def test_buffers_that_do_not_fit_are_refused():
    x, w, y = (torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV) for _ in range(3))
    call = lambda x=x, w=w, y=y, z=None, e=False: F.flashdp_linear_forward(x, w, None, None, 8, 16, 8, F.BF16, None, y, z, e)    # noqa: E731
    call()
    for bad in (dict(x=torch.zeros(16, 8, dtype=torch.bfloat16, device=DEV).t()), dict(x=x[:4]), dict(x=x.float()), dict(y=y[:2]), dict(w=w[:, ::2]), dict(x=x.cpu()),
                dict(z=torch.zeros(10, dtype=torch.uint8, device=DEV), e=True), dict(z=y, e=True)):
        with pytest.raises(F.FlashDPError):
            call(**bad)
    n = torch.zeros(8, device=DEV)
    with pytest.raises(F.FlashDPError):
        F.flashdp_layernorm_forward(x, w[0], None, 8, 16, F.BF16, 1e-5, y, n[:4], n)
    with pytest.raises(F.FlashDPError):      # a view that starts between two 16-byte boundaries
        call(x=torch.zeros(200, dtype=torch.bfloat16, device=DEV)[1:129].view(8, 16))


def test_the_library_workspace_is_not_taken_by_a_graph():
    """Large enough or not: a graph would keep its address past the call that grows it."""
    dy, x, g = torch.randn(2, 40, 64, device=DEV), torch.randn(2, 40, 64, device=DEV), torch.zeros(64, device=DEV)
    gam, mean, gn = torch.ones(64, device=DEV), torch.zeros(80, device=DEV), torch.zeros(2, 64, device=DEV)
    packed = torch.zeros(F.flashdp_checkpoint8_bytes(80, 64), dtype=torch.uint8, device=DEV)
    L = [dict(X=packed, dY=dy, d_in=64, d_out=64, C=1.0, sigma=0.0, seed=0, layer=0, out_grad=torch.zeros(64, 64, device=DEV), out_norms=None)]
    calls = [lambda: F.flashdp_activation_dp_grad(dy, None, False, 2, 40, 64, F.F32, None, 1.0, 0.0, 0, 0, None, g),
             lambda: F.flashdp_layernorm_dp_grad(x, dy, gam, mean, mean, 2, 40, 64, F.F32, 1.0, 0.0, 0, 0, None, gn),
             lambda: F.flashdp_block_dp_grad_checkpoint8(L, 2, 40, F.F32, "twopass")]
    for call in calls:
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in calls:
            with pytest.raises(F.FlashDPError) as e:
                call()
            assert e.value.status == F.WORKSPACE_TOO_SMALL
        g.add_(1.0)
    del graph
    for call in calls:
        call()
    torch.cuda.synchronize()


# ---- offsets that pass 32 bits ----------------------------------------------------------------------

LONG = (1100000, 2048)      # rows and features: 2.25e9 elements, 4.5 GB in 16 bits
LOOK = [0, 1, 524287, 524288, 1048575, 1048576, 1099990, 1099999]      # rows on both sides of 2^30 and 2^31 elements, and the last


def long_rows(d=LONG[1], rows=LONG[0]):
    return torch.empty(rows, d, dtype=torch.bfloat16, device=DEV).normal_()


@pytest.mark.parametrize("K,D", [(2048, 40), (40, 2048), (2047, 24), (24, 2047)])
def test_forward_of_long_inputs(K, D):
    """Tolerance: one rounding to bfloat16 and fp32 sums of at most 2048 products."""
    rows = LONG[0]
    x, w, y = long_rows(K), torch.randn(D, K, device=DEV).bfloat16(), torch.empty(rows, D, dtype=torch.bfloat16, device=DEV)
    F.flashdp_linear_forward(x, w, None, None, rows, K, D, F.BF16, None, y)
    torch.cuda.synchronize()
    x64, w64 = x[LOOK].cpu().double(), w.cpu().double()
    want, size = x64 @ w64.T, x64.abs() @ w64.abs().T
    assert bool(((y[LOOK].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + K * 2.0 ** -24 * size).all())


def test_normalisation_of_long_inputs():
    """Forward and dX on the rows looked at: fp32 sums of 2048 terms and one rounding; the parameters' gradients against sums in 64 bits over all rows.  Those are
    fp32 sums of 2^12 terms at most in a row, so off by less than 2^-12 of the sum of magnitudes; a row read elsewhere moves them by more."""
    B, (rows, d) = 2, LONG
    T = rows // B
    x, dy = long_rows(), long_rows()
    gam, bet = torch.randn(d, device=DEV).bfloat16(), torch.randn(d, device=DEV).bfloat16()
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, g, n = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(2, d, device=DEV), torch.empty(B, device=DEV)
    F.flashdp_layernorm_forward(x, gam, bet, rows, d, F.BF16, 1e-5, y, mean, rstd)
    F.flashdp_layernorm_dp_grad(x, dy, gam, mean, rstd, B, T, d, F.BF16, 1e6, 0.0, 0, 0, dx, g, n)
    torch.cuda.synchronize()
    x64, dy64, g64, b64 = x[LOOK].cpu().double(), dy[LOOK].cpu().double(), gam.cpu().double(), bet.cpu().double()
    mu = x64.mean(1, keepdim=True)
    r = ((x64 - mu).square().mean(1, keepdim=True) + 1e-5) ** -0.5
    xh, a = (x64 - mu) * r, dy64 * g64
    dx64 = r * (a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True))
    for got, want in ((y[LOOK], xh * g64 + b64), (dx[LOOK], dx64)):
        assert bool(((got.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-3 * 2.0 ** -8 * want.abs().max()).all())
    del y, dx
    total, size, norms = torch.zeros(2, d, device=DEV, dtype=torch.float64), torch.zeros(2, d, device=DEV, dtype=torch.float64), []
    for i in range(B):
        s = torch.zeros(2, d, device=DEV, dtype=torch.float64)
        for k in range(i * T, (i + 1) * T, 50000):
            e = min(k + 50000, (i + 1) * T)
            dyk = dy[k:e].double()
            p = dyk * ((x[k:e].double() - mean[k:e, None].double()) * rstd[k:e, None].double())
            s += torch.stack((p.sum(0), dyk.sum(0)))
            size += torch.stack((p.abs().sum(0), dyk.abs().sum(0)))
        total += s
        norms.append(float(s.norm()))
    assert bool(((g.double() - total).abs() <= 2.0 ** -12 * size).all())
    for got, want in zip(n.tolist(), norms):
        assert abs(got - want) <= 1e-3 * want


def test_activation_gradient_and_checkpoints_of_long_inputs():
    """dZ from a checkpoint of Z (ReLU: exact), the bias's gradient as in the test above, and the checkpoint's way back."""
    B, (rows, d) = 2, LONG
    T = rows // B
    z, dy = long_rows(), long_rows()
    packed, back = torch.empty(F.flashdp_checkpoint8_bytes(rows, d), dtype=torch.uint8, device=DEV), torch.empty_like(z)
    F.flashdp_checkpoint8_pack(z, rows, d, F.BF16, packed)
    F.flashdp_checkpoint8_unpack(packed, rows, d, F.BF16, back)
    torch.cuda.synchronize()
    assert torch.equal(back[LOOK].cpu().double(), quantise(z[LOOK].cpu().double(), False)[2])
    dz, g, n = z, torch.empty(d, device=DEV), torch.empty(B, device=DEV)
    F.flashdp_activation_dp_grad(dy, packed, True, B, T, d, F.BF16, "relu", 1e6, 0.0, 0, 0, dz, g, n)
    torch.cuda.synchronize()
    total, size = torch.zeros(d, device=DEV, dtype=torch.float64), torch.zeros(d, device=DEV, dtype=torch.float64)
    for k in range(0, rows, 50000):
        want = torch.where(back[k:k + 50000] > 0, dy[k:k + 50000], torch.zeros((), dtype=dy.dtype, device=DEV))
        assert torch.equal(dz[k:k + 50000], want), k
        total += want.double().sum(0)
        size += want.double().abs().sum(0)
    assert bool(((g.double() - total).abs() <= 2.0 ** -12 * size).all())
