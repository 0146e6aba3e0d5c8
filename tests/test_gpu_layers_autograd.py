"""The layers as modules: gradients of a block of them against the definition in 64 bits, sample by sample, and the
bookkeeping of noise, steps and deferred weight gradients."""
import math

import numpy as np
import pytest
import torch

import paper_2507_01154_amd as F
from oracle import flashdp_oracle as O
from gpu_util import DEV
from test_gpu_layers import act64, clipped64, quantise

pytestmark = pytest.mark.gpu


def modules(dtype, d, ff, checkpoint, sigma=0.0, C=1.0, **kw):
    from paper_2507_01154_amd.autograd import DPLayerNorm, DPLinear
    torch.manual_seed(5)
    common = dict(C=C, sigma=sigma, seed=9, dtype=dtype, device=DEV, keep_fp32_grad=True, auto_step=False)
    ln = DPLayerNorm(d, layer=0, **common)
    up = DPLinear(d, ff, layer=1, bias=True, activation="gelu_tanh", checkpoint=checkpoint, schedule="twopass", **common, **kw)
    down = DPLinear(ff, d, layer=2, bias=True, checkpoint=checkpoint, schedule="twopass", **common, **kw)
    with torch.no_grad():
        for p in (ln.weight, ln.bias, up.bias, down.bias):
            p.add_(0.1 * torch.randn_like(p))
    return ln, up, down


def block(ln, up, down, x):
    return down(up(ln(x)), residual=x)


@pytest.mark.parametrize("T", [1, 37])
@pytest.mark.parametrize("checkpoint", [None, "8bit"])
def test_mlp_block_gradients_are_the_definitions(T, checkpoint):
    """fp32: y = x + down(gelu(up(ln(x)))) on a loss <dY, y>, every parameter's clipped sum against 64 bits; with 8-bit
    checkpoints at the kept values.  What separates the two are fp32 sums of at most 256 terms: a relative 1e-4 of the norm is
    more than 20 times their error, and the 8-bit kept values themselves may move by a step where a sum lies on a
    border, 2^-7 of the largest of 32 for one element in ten thousand."""
    B, d, ff = 5, 72, 200
    ln, up, down = modules(torch.float32, d, ff, checkpoint)
    x = torch.randn(B, T, d, device=DEV)
    dy = torch.randn(B, T, d, device=DEV) * torch.logspace(-1.5, 1, B, device=DEV)[:, None, None]
    x.requires_grad_(True)
    y = block(ln, up, down, x)
    y.backward(dy)
    torch.cuda.synchronize()
    c = lambda t: t.detach().cpu().double()     # noqa: E731
    x64, dy64 = c(x).view(-1, d), c(dy).view(-1, d)
    mu = x64.mean(1, keepdim=True)
    r = ((x64 - mu).square().mean(1, keepdim=True) + ln.eps) ** -0.5
    xh = (x64 - mu) * r
    h = xh * c(ln.weight) + c(ln.bias)
    z = h @ c(up.weight).T + c(up.bias)
    a = act64(z, "gelu_tanh")[0]
    y64 = x64 + a @ c(down.weight).T + c(down.bias)
    kept = (lambda t: quantise(t, False)[2]) if checkpoint else (lambda t: t)
    da = dy64 @ c(down.weight)
    dz = da * act64(kept(z), "gelu_tanh")[1]
    dh = dz @ c(up.weight)
    p = dh * c(ln.weight)
    dx = dy64 + r * (p - p.mean(1, keepdim=True) - xh * (p * xh).mean(1, keepdim=True))
    s = lambda t: t.view(B, T, -1)      # noqa: E731
    outer = lambda g, v: (s(g).transpose(1, 2) @ s(v)).reshape(B, -1)      # noqa: E731
    want = {"ln": torch.cat((s(dh * xh).sum(1), s(dh).sum(1)), 1), "up_b": s(dz).sum(1), "down_b": s(dy64).sum(1),
            "up": outer(dz, kept(h)), "down": outer(dy64, kept(a))}
    got = {"ln": (ln.grad_fp32, ln.last_norms), "up_b": (up.bias_grad_fp32, up.last_bias_norms), "down_b": (down.bias_grad_fp32, down.last_bias_norms),
           "up": (up.grad_fp32, up.last_norms), "down": (down.grad_fp32, down.last_norms)}
    tol = 1e-3 if checkpoint else 1e-4
    assert float((c(y).view(-1, d) - y64).norm() / y64.norm()) <= 1e-5
    assert float((c(x.grad).view(-1, d) - dx).norm() / dx.norm()) <= tol
    for k, G in want.items():
        out, norms, fac = clipped64(G, 1.0, 0.0, 0, 0, 0)
        assert float((c(got[k][0]).reshape(-1) - out).norm() / out.norm()) <= tol, k
        assert float(((c(got[k][1]) - norms) / norms).abs().max()) <= tol, k
        if T > 1:
            assert bool((fac < 1).any()), k
    assert torch.equal(up.weight.grad, up.grad_fp32) and torch.equal(ln.bias.grad, ln.grad_fp32[1]) and torch.equal(down.bias.grad, down.bias_grad_fp32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_sixteen_bit_block_is_near_the_single_precision_one(dtype):
    """The same block in 16 bits, 8-bit checkpoints: gradients within the roundings on their way (a dozen at half a step of
    the type each, at most 2^-8, and 8-bit values off by a 64th of their block's largest at worst, a 300th in the mean)."""
    B, T, d, ff = 4, 40, 128, 256
    exact, low = modules(torch.float32, d, ff, None, C=1e6), modules(dtype, d, ff, "8bit", C=1e6)
    with torch.no_grad():
        for m, n in zip(low, exact):
            for p, q in zip(m.parameters(), n.parameters()):
                q.copy_(p)
    x, dy = torch.randn(B, T, d, device=DEV).to(dtype), torch.randn(B, T, d, device=DEV).to(dtype)
    block(*exact, x.float()).backward(dy.float())
    block(*low, x).backward(dy)
    for m, n in zip(low, exact):
        for p, q in zip(m.parameters(), n.parameters()):
            assert p.grad.dtype == dtype and float((p.grad.float() - q.grad).norm() / q.grad.norm()) <= 0.03
        assert float(((m.last_norms - n.last_norms) / n.last_norms).abs().max()) <= 0.03


def test_deferred_weight_gradients_from_checkpoints():
    from paper_2507_01154_amd.autograd import DPLinear, deferred_weight_grads
    ms = modules(torch.bfloat16, 128, 256, "8bit", sigma=0.5)
    plain = DPLinear(128, 64, sigma=0.5, seed=9, layer=7, dtype=torch.bfloat16, device=DEV, auto_step=False, schedule="twopass")
    x, dy = torch.randn(3, 50, 128, device=DEV).bfloat16(), torch.randn(3, 50, 64, device=DEV).bfloat16()

    def run():
        for m in (*ms, plain):
            for p in m.parameters():
                p.grad = None
        plain(block(*ms, x)).backward(dy)

    run()
    want = [p.grad.clone() for m in (*ms, plain) for p in m.parameters()]
    with deferred_weight_grads("twopass"):
        run()
        assert ms[1].weight.grad is None and plain.weight.grad is None and ms[1].bias.grad is not None
    got = [p.grad for m in (*ms, plain) for p in m.parameters()]
    for a, b in zip(got, want):
        assert float((a.float() - b.float()).norm() / b.float().norm()) <= 2.0 ** -8


def test_noise_differs_between_parameters_and_steps_and_goes_in_once():
    from paper_2507_01154_amd.autograd import DPLayerNorm, DPLinear
    kw = dict(C=2.0, sigma=0.5, seed=4, layer=3, dtype=torch.float32, device=DEV, keep_fp32_grad=True)
    lin, ln = DPLinear(16, 24, bias=True, bias_C=3.0, schedule="twopass", **kw), DPLayerNorm(24, **kw)
    x = torch.randn(4, 6, 16, device=DEV)
    fields = []
    for step in range(2):
        for m in (lin, ln):
            m.zero_fp32_grad()
        ln(lin(x)).backward(torch.zeros(4, 6, 24, device=DEV))          # no signal: what comes back is the noise
        seed = lin.last_seed
        assert seed == 4 + (step << 32) and lin.step == step + 1 and ln.last_seed == seed
        zero = lambda n: torch.zeros(1, n, dtype=torch.float64)     # noqa: E731
        for got, n, C, field in ((lin.grad_fp32, 384, 2.0, 0), (lin.bias_grad_fp32, 24, 3.0, F.FIELD_BIAS), (ln.grad_fp32, 48, 2.0, F.FIELD_NORM)):
            want = clipped64(zero(n), C, 0.5, seed, 3, field)[0]
            assert float((got.cpu().double().reshape(-1) - want).abs().max()) <= 2e-6 * C
            fields.append(want[:24])
    for i in range(6):
        for j in range(i):
            assert float((fields[i] / fields[i].norm() @ (fields[j] / fields[j].norm())).abs()) < 0.9
    # micro-batches: noise with the last one only
    for m in (lin, ln):
        m.zero_fp32_grad()
        m.add_noise = False
    ln(lin(x[:2])).backward(torch.zeros(2, 6, 24, device=DEV))
    assert float(lin.bias_grad_fp32.abs().max()) == 0.0 and float(ln.grad_fp32.abs().max()) == 0.0 and lin.step == 2


def test_frozen_parameters_no_grad_and_inputs_of_other_layouts():
    from paper_2507_01154_amd.autograd import DPLayerNorm, DPLinear
    kw = dict(C=1.0, sigma=0.0, dtype=torch.bfloat16, device=DEV)
    lin, ln = DPLinear(40, 24, bias=True, activation="silu", checkpoint="8bit", **kw), DPLayerNorm(40, **kw)
    x = torch.randn(6, 40, 5, device=DEV).bfloat16().transpose(1, 2)            # [6, 5, 40], rows not one after the other
    ref = lin(ln(x.contiguous()))
    assert torch.equal(lin(ln(x)), ref) and ref.shape == (6, 5, 24)
    odd = torch.empty(6 * 5 * 40 + 1, device=DEV, dtype=torch.bfloat16)[1:].view(6, 5, 40)      # starts between two 16-byte boundaries
    odd.copy_(x)
    assert torch.equal(lin(ln(odd)), ref)
    with torch.no_grad():
        y = lin(ln(x))
    assert torch.equal(y, ref) and y.grad_fn is None
    lin.weight.requires_grad_(False)
    ln.weight.requires_grad_(False)
    xg = x.detach().contiguous().requires_grad_(True)
    lin(ln(xg)).sum().backward()
    assert lin.weight.grad is None and ln.weight.grad is None and lin.bias.grad is not None and ln.bias.grad is not None and xg.grad.shape == xg.shape
    with pytest.raises(TypeError):
        lin(x.float())
    with pytest.raises(TypeError):
        lin(x, residual=x)
    with pytest.raises(TypeError):
        ln(x.float())


def test_layers_without_an_epilogue_take_the_path_they_took():
    from paper_2507_01154_amd.autograd import DPLinear
    torch.manual_seed(1)
    lin = DPLinear(64, 40, C=1.0, sigma=0.0, device=DEV)
    x = torch.randn(3, 20, 64, device=DEV).bfloat16()
    assert torch.equal(lin(x), torch.matmul(x, lin.weight.t()))


@pytest.mark.parametrize("checkpoint", [None, "8bit"])
def test_a_captured_step_gives_what_an_eager_one_gives(checkpoint):
    """Forward and backward pass in a graph, replayed beside eager work that makes the library's workspace grow.  The captured modules are never
    run eagerly."""
    eager, captured = (modules(torch.bfloat16, 64, 96, checkpoint, sigma=0.5) for _ in range(2))
    for a, b in zip(eager, captured):
        a.keep_fp32_grad = b.keep_fp32_grad = False
        a.load_state_dict(b.state_dict())
    x, dy = torch.empty(3, 40, 64, device=DEV, dtype=torch.bfloat16), torch.empty(3, 40, 64, device=DEV, dtype=torch.bfloat16)

    def step(ms):
        ps = [p for m in ms for p in m.parameters() if p.requires_grad]
        return torch.autograd.grad(block(*ms, x), ps, dy)

    def draw(seed):
        torch.manual_seed(seed)
        x.normal_()
        dy.normal_()

    draw(1)
    want = [t.clone() for t in step(eager)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(captured)
    for rep in range(3):
        draw(rep)
        want = [t.clone() for t in step(eager)]
        big = 256 << rep                     # a larger layer each time
        o = torch.empty(big, big, device=DEV)
        a = torch.ones(2, 64, big, device=DEV, dtype=torch.bfloat16)
        F.flashdp_block_dp_grad([dict(X=a, dY=a, d_in=big, d_out=big, C=1.0, sigma=0.0, seed=0, layer=0, out_grad=o)], 2, 64, F.BF16, "scratch")
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w), rep
