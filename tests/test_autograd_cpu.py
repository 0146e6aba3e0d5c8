"""The modules' glue on the CPU: what is recorded, deferred, refused and handed on, with the library's calls replaced by the
formulas in torch.  The library's own arithmetic is tested on the GPU."""
import contextlib

import pytest
import torch

from paper_2507_01154_amd import autograd as A


def clipped(G, C):
    """sum_i G_i / max(1, |G_i| / C) and the norms, of per-sample gradients G [B, ...]."""
    n = G.reshape(G.shape[0], -1).norm(dim=1)
    return (G / (n / C).clamp(min=1.0).reshape(-1, *(1,) * (G.dim() - 1))).sum(0), n


class Calls(list):
    def __init__(self):
        super().__init__()
        self.rooms = []


@pytest.fixture
def library(monkeypatch):
    """The calls that the modules make, in torch, without noise, activations or 8-bit forms.  `calls` lists the block calls: layers and noise flag;
    calls.rooms their workspaces."""
    calls = Calls()

    def linear_forward(X, W, bias, residual, rows, d_in, d_out, dtype, activation, Y, Z=None, z_8bit=False, stream=None):
        y = X.reshape(rows, d_in) @ W.t()
        y = y if bias is None else y + bias
        Y.reshape(rows, d_out).copy_(y if residual is None else y + residual.reshape(rows, d_out))

    def activation_grad(dY, Z, z_8bit, B, T, d_out, dtype, activation, C, sigma, seed, layer, dZ, out_grad, out_norms=None, workspace=None, stream=None,
                        accumulate=False, add_noise=True):
        g, n = clipped(dY.reshape(B, T, d_out).sum(1), C)
        out_grad.copy_(g)
        out_norms.copy_(n)

    def block(layers, B, T, dtype, schedule="auto", workspace=None, stream=None, accumulate=False, add_noise=True):
        calls.append((len(layers), add_noise))
        calls.rooms.append(workspace)
        for L in layers:
            G = L["dY"].reshape(B, T, -1).transpose(1, 2) @ L["X"].reshape(B, T, -1)
            g, n = clipped(G, L["C"])
            L["out_grad"].copy_(g)
            if L["out_norms"] is not None:
                L["out_norms"].copy_(n)

    def norm_forward(X, gamma, beta, rows, d, dtype, eps, Y, mean=None, rstd=None, stream=None):
        Y.copy_(torch.nn.functional.layer_norm(X, (d,), gamma, beta, eps))

    def norm_grad(X, dY, gamma, mean, rstd, B, T, d, dtype, C, sigma, seed, layer, dX, out_grad, out_norms=None, bias=True, workspace=None, stream=None,
                  accumulate=False, add_noise=True):
        out_grad.zero_()
        if dX is not None:
            dX.copy_(dY)

    for name, f in (("flashdp_linear_forward", linear_forward), ("flashdp_activation_dp_grad", activation_grad), ("flashdp_block_dp_grad_micro", block),
                    ("flashdp_layernorm_forward", norm_forward), ("flashdp_layernorm_dp_grad", norm_grad)):
        monkeypatch.setattr(A.F, name, f)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return calls


def linear(d_in=6, d_out=4, **kw):
    torch.manual_seed(3)
    return A.DPLinear(d_in, d_out, **dict(dict(C=1.0, sigma=0.0, device="cpu", dtype=torch.float32, auto_step=False), **kw))


@pytest.mark.parametrize("bias", [False, True])
def test_a_leaf_residual_and_two_backward_passes_inside_one_deferred_context(library, bias):
    """The output's gradient goes to the residual as it is, and is a deferred layer's dY: adding to residual.grad must not reach it."""
    torch.manual_seed(1)
    xs, dys = [torch.randn(3, 5, 6) for _ in range(2)], [torch.randn(3, 5, 4) for _ in range(2)]
    got = []
    for deferred in (False, True):
        lin, r = linear(bias=bias), torch.randn(3, 5, 4, generator=torch.Generator().manual_seed(2)).requires_grad_()
        with A.deferred_weight_grads() if deferred else contextlib.nullcontext():
            for x, dy in zip(xs, dys):
                # (clone: the passes' gradients are made on their way, as they are inside a model, and nobody else holds them)
                (lin(x, residual=r) * 2.0).backward(dy.clone())
            r.grad.mul_(3.0)
        got.append([r.grad, lin.weight.grad] + ([lin.bias.grad] if bias else []))
    for a, b in zip(*got):
        assert torch.allclose(a, b, rtol=1e-6, atol=1e-6)
    want = sum(clipped((2.0 * dy).transpose(1, 2) @ x, 1.0)[0] for x, dy in zip(xs, dys))
    assert torch.allclose(got[1][1], want, rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("epilogue", [False, True])
@pytest.mark.parametrize("which", ["input", "gradient"])
def test_what_a_deferred_layer_was_recorded_with_is_not_written_before_the_context_ends(library, which, epilogue):
    """As autograd does for what it saves: a buffer that the next micro-batch is copied into would give gradients of the wrong samples."""
    lin, x, dy = linear(bias=epilogue), torch.randn(3, 5, 6), torch.randn(3, 5, 4)
    with pytest.raises(RuntimeError, match="in place"):
        with A.deferred_weight_grads():
            lin(x).backward(dy)
            (x if which == "input" else dy).normal_()
    assert lin.weight.grad is None and library == []
    with A.deferred_weight_grads():          # and the next context starts empty
        lin(x).backward(dy)
    assert library == [(1, True)] and torch.allclose(lin.weight.grad, clipped(dy.transpose(1, 2) @ x, 1.0)[0], rtol=1e-5, atol=1e-6)
    with A.deferred_weight_grads():          # afterwards they are the caller's
        lin(x).backward(dy)
    x.zero_()
    dy.zero_()


def test_deferred_layers_of_two_devices_go_to_two_calls_each_on_its_own_device(library, monkeypatch):
    """Equal shapes on two devices ("meta" standing for the second): the library works on the current device."""
    entered = []
    monkeypatch.setattr(torch.cuda, "device", lambda d: entered.append(torch.device(d).type) or contextlib.nullcontext())
    layers = [linear(), linear(device="meta"), linear()]
    with A.deferred_weight_grads():
        for lin in layers:
            x = torch.ones(3, 5, 6, device=lin.weight.device)
            lin(x).backward(torch.ones(3, 5, 4, device=x.device))
        del entered[:]
    assert library == [(2, True), (1, True)] and entered == ["cpu", "meta"]
    assert all(lin.weight.grad.device == lin.weight.device for lin in layers) and torch.equal(layers[0].weight.grad, layers[2].weight.grad)


def test_a_graph_does_not_capture_noise_that_its_replays_would_repeat(library, monkeypatch):
    """The step advances in Python and the seed goes by value, so a replay would add the field of the capture again.  Modules that promise another
    field every step refuse; without noise, or with the step left to the caller, they are captured."""
    def backward(m):
        x = torch.randn(3, 5, 6)
        m(x).backward(torch.randn(3, 5, m.weight.shape[0]))

    norm = lambda **kw: A.DPLayerNorm(6, device="cpu", dtype=torch.float32, **kw)      # noqa: E731
    makers = [lambda **kw: linear(**kw), lambda **kw: linear(bias=True, **kw), norm]
    for make in makers:
        refused, quiet, by_hand, micro = make(sigma=0.5, auto_step=True), make(sigma=0.0, auto_step=True), make(sigma=0.5, auto_step=False), make(sigma=0.5, auto_step=True)
        micro.add_noise = False
        for capturing in (False, True):
            monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
            for m in (quiet, by_hand, micro):
                backward(m)
            if not capturing:
                backward(refused)
                continue
            for p in refused.parameters():
                p.grad = None
            with pytest.raises(RuntimeError, match="replay"):
                backward(refused)
            assert all(p.grad is None for p in refused.parameters())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    frozen = linear(sigma=0.5, auto_step=True, bias=True)      # no parameter of it is trained: no noise
    for p in frozen.parameters():
        p.requires_grad_(False)
    x = torch.randn(3, 5, 6, requires_grad=True)
    frozen(x).backward(torch.ones(3, 5, 4))
    lin = linear(sigma=0.5, auto_step=True)
    with pytest.raises(RuntimeError, match="replay"):
        with A.deferred_weight_grads():
            backward(lin)
    assert lin.weight.grad is None
    with A.deferred_weight_grads():      # recorded in the capture, computed after it: once
        backward(lin)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    assert lin.weight.grad is not None


def test_a_captured_backward_pass_never_takes_the_librarys_workspace(library, monkeypatch):
    """A graph keeps the addresses of its capture, and the library's workspace moves when a later call makes it grow: every kind of layer, alone or
    deferred, brings memory of torch's, which the graph keeps, where it is captured."""
    def pass_of(deferred, T):
        with A.deferred_weight_grads() if deferred else contextlib.nullcontext():
            for m in layers:
                x = torch.randn(3, T, 6)
                m(x, residual=torch.zeros(3, T, 4) if m.bias is not None else None).backward(torch.randn(3, T, 4))

    layers = [linear(), linear(bias=True), linear()]
    for capturing in (False, True):
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
        for deferred in (False, True):
            for T in (1, 5):
                del library[:], library.rooms[:]
                pass_of(deferred, T)
                assert [n for n, _ in library] == ([3] if deferred else [1, 1, 1])
                assert all((r is not None) == capturing for r in library.rooms)
                for r in library.rooms if capturing else []:
                    # what any schedule needs at least; with a sequence, what the layers park in, twice where one can be summed beside the next
                    size = lambda s: A.F.flashdp_workspace_bytes([dict(X=None, dY=None, d_in=6, d_out=4, C=1.0, sigma=0.0, seed=0, layer=0, out_grad=None)] * 3, 3, T, A.F.F32, s)   # noqa: E731
                    assert r.numel() >= size("twopass" if T == 1 else "overlap" if deferred else "scratch")
