"""CPU-side checks of the layers around the weight gradient: what is refused before a device is touched, the sizing calls, the
Python layer's own checks, and the register use of the kernels.  No kernel is launched here."""
import os
import re
import subprocess

import pytest
import torch

import paper_2507_01154_amd as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, B_, C_, D_, E_ = 0x10000, 0x20000, 0x30000, 0x40000, 0x50000      # fake, aligned, never dereferenced
INV, MIS, SHAPE, SMALL = F.INVALID_ARGUMENT, F.MISALIGNED, F.UNSUPPORTED_SHAPE, F.WORKSPACE_TOO_SMALL
INF, NAN = float("inf"), float("nan")


def refused(name, good, changes, want):
    args = dict(good)
    args.update(changes)
    assert getattr(F.lib(), name)(*args.values()) == want, (name, changes)


FORWARD = dict(X=A, W=B_, bias=None, residual=None, rows=4, d_in=8, d_out=8, dtype=0, act=0, Y=C_, Z=None, z_8bit=0, stream=None)


@pytest.mark.parametrize("changes,want", [
    (dict(X=None), INV), (dict(W=None), INV), (dict(Y=None), INV), (dict(dtype=3), INV), (dict(dtype=-1), INV), (dict(act=5), INV), (dict(act=-1), INV),
    (dict(z_8bit=2, Z=D_), INV), (dict(z_8bit=1), INV), (dict(rows=0), INV), (dict(d_in=0), INV), (dict(d_out=-1), INV),
    (dict(X=A + 8), MIS), (dict(W=B_ + 2), MIS), (dict(bias=D_ + 4), MIS), (dict(residual=D_ + 8), MIS), (dict(Y=C_ + 1), MIS), (dict(Z=D_ + 8), MIS),
    (dict(rows=1 << 40), SHAPE), (dict(d_in=(1 << 30) + 1), SHAPE), (dict(d_out=(1 << 30) + 1), SHAPE), (dict(rows=1 << 38), SHAPE),
    (dict(rows=1 << 30, d_out=1 << 20), SHAPE), (dict(rows=1 << 30, d_in=9, d_out=1 << 20), SHAPE)])
def test_forward_refuses(changes, want):
    refused("flashdp_linear_forward", FORWARD, changes, want)


ACTIVATION = dict(dY=A, Z=B_, z_8bit=0, B=2, T=4, d=8, dtype=0, act=1, C=1.0, sigma=0.0, seed=0, layer=0, dZ=C_, out=D_, norms=E_, ws=None, bytes=0,
                  stream=None, accumulate=0, noise=1)


@pytest.mark.parametrize("changes,want", [
    (dict(dY=None), INV), (dict(Z=None), INV), (dict(dZ=None, out=None), INV), (dict(act=9), INV), (dict(dtype=7), INV), (dict(z_8bit=3), INV),
    (dict(C=0.0), INV), (dict(C=-1.0), INV), (dict(C=NAN), INV), (dict(C=INF), INV), (dict(sigma=-1.0), INV), (dict(sigma=NAN), INV),
    (dict(B=0), INV), (dict(T=0), INV), (dict(d=0), INV), (dict(T=-1), INV), (dict(dY=A + 4), MIS), (dict(Z=B_ + 8), MIS), (dict(dZ=C_ + 2), MIS),
    (dict(out=D_ + 4), MIS), (dict(norms=E_ + 2), MIS), (dict(ws=A + 8, bytes=1 << 20), MIS), (dict(ws=A, bytes=16), SMALL),
    (dict(B=1 << 20), SHAPE), (dict(T=1 << 31), SHAPE), (dict(d=(1 << 30) + 1), SHAPE)])
def test_activation_refuses(changes, want):
    refused("flashdp_activation_dp_grad", ACTIVATION, changes, want)


NORM = dict(X=A, gamma=B_, beta=C_, rows=4, d=8, dtype=0, eps=1e-5, Y=D_, mean=E_, rstd=E_, stream=None)


@pytest.mark.parametrize("changes,want", [
    (dict(X=None), INV), (dict(gamma=None), INV), (dict(Y=None), INV), (dict(eps=0.0), INV), (dict(eps=-1e-5), INV), (dict(eps=NAN), INV), (dict(eps=INF), INV),
    (dict(dtype=4), INV), (dict(rows=0), INV), (dict(d=0), INV), (dict(X=A + 2), MIS), (dict(gamma=B_ + 4), MIS), (dict(beta=C_ + 8), MIS), (dict(Y=D_ + 2), MIS),
    (dict(mean=E_ + 1), MIS), (dict(rstd=E_ + 2), MIS), (dict(rows=1 << 31), SHAPE), (dict(d=1 << 31), SHAPE)])
def test_layernorm_refuses(changes, want):
    refused("flashdp_layernorm_forward", NORM, changes, want)


NORM_GRAD = dict(X=A, dY=B_, gamma=C_, mean=E_, rstd=E_, B=2, T=4, d=8, dtype=0, C=1.0, sigma=0.0, seed=0, layer=0, dX=D_, out=D_, norms=E_, bias=1, ws=None,
                 bytes=0, stream=None, accumulate=0, noise=1)


@pytest.mark.parametrize("changes,want", [
    (dict(X=None), INV), (dict(dY=None), INV), (dict(gamma=None), INV), (dict(mean=None), INV), (dict(rstd=None), INV), (dict(dX=None, out=None), INV),
    (dict(C=0.0), INV), (dict(sigma=INF), INV), (dict(dtype=-2), INV), (dict(B=-1), INV), (dict(T=0), INV), (dict(d=0), INV), (dict(X=A + 8), MIS), (dict(dY=B_ + 8), MIS),
    (dict(gamma=C_ + 8), MIS), (dict(mean=E_ + 2), MIS), (dict(rstd=E_ + 2), MIS), (dict(dX=D_ + 8), MIS), (dict(out=D_ + 8), MIS), (dict(norms=E_ + 2), MIS),
    (dict(ws=A + 4, bytes=1 << 20), MIS), (dict(ws=A, bytes=64), SMALL), (dict(B=1 << 20), SHAPE), (dict(d=1 << 31), SHAPE)])
def test_layernorm_gradient_refuses(changes, want):
    refused("flashdp_layernorm_dp_grad", NORM_GRAD, changes, want)


@pytest.mark.parametrize("name", ["flashdp_checkpoint8_pack", "flashdp_checkpoint8_unpack"])
@pytest.mark.parametrize("changes,want", [
    (dict(a=None), INV), (dict(b=None), INV), (dict(dtype=3), INV), (dict(rows=0), INV), (dict(d=0), INV), (dict(a=A + 8), MIS), (dict(b=B_ + 4), MIS),
    (dict(rows=1 << 40), SHAPE), (dict(rows=1 << 39, d=64), SHAPE), (dict(d=1 << 31), SHAPE)])
def test_checkpoints_refuse(name, changes, want):
    refused(name, dict(a=A, rows=4, d=8, dtype=0, b=B_, stream=None), changes, want)


@pytest.mark.parametrize("changes,call,want", [
    ({}, dict(n=0), INV), ({}, dict(dtype=3), INV), ({}, dict(schedule=7), INV), ({}, dict(schedule=-1), INV), ({}, dict(B=0), INV), ({}, dict(T=-1), INV),
    (dict(X=None), {}, INV), (dict(dY=None), {}, INV), (dict(out_grad=None), {}, INV), (dict(C=0.0), {}, INV), (dict(sigma=NAN), {}, INV), (dict(d_in=0), {}, INV),
    (dict(d_out=-8), {}, INV), (dict(X=A + 8), {}, MIS), (dict(dY=A + 2), {}, MIS), (dict(out_grad=A + 4), {}, MIS), (dict(out_norms=A + 1), {}, MIS),
    ({}, dict(ws=A + 8, bytes=1 << 30), MIS), ({}, dict(ws=A, bytes=4), SMALL), ({}, dict(T=1 << 30), SHAPE), ({}, dict(B=1 << 20), SHAPE)])
def test_gradient_from_checkpoints_refuses(changes, call, want):
    arr = (F.flashdp_layer_t * 1)()
    for k, v in dict(dict(X=A, dY=B_, d_in=8, d_out=8, C=1.0, sigma=0.0, seed=0, layer=0, out_grad=C_, out_norms=D_), **changes).items():
        setattr(arr[0], k, v)
    c = dict(dict(n=1, B=2, T=4, dtype=0, schedule=1, ws=None, bytes=0, stream=None, accumulate=0, noise=1), **call)
    assert F.lib().flashdp_block_dp_grad_checkpoint8(arr, *c.values()) == want
    assert F.lib().flashdp_block_dp_grad_checkpoint8(None, 1, 2, 4, 0, 1, None, 0, None, 0, 1) == INV


@pytest.mark.skipif(torch.cuda.is_available(), reason="only meaningful on a host without a GPU")
def test_no_device_is_an_error():
    for name, good in (("flashdp_linear_forward", FORWARD), ("flashdp_activation_dp_grad", ACTIVATION), ("flashdp_layernorm_forward", NORM),
                       ("flashdp_layernorm_dp_grad", NORM_GRAD)):
        refused(name, good, {}, F.NO_DEVICE)
    assert F.lib().flashdp_checkpoint8_pack(A, 4, 8, 0, B_, None) == F.NO_DEVICE


def test_sizing_calls():
    assert F.flashdp_checkpoint8_bytes(1, 1) == 16 + 1 and F.flashdp_checkpoint8_bytes(3, 33) == 112 + 6
    assert F.flashdp_checkpoint8_bytes(2, 64) == 128 + 4 and F.flashdp_checkpoint8_bytes(0, 4) == 0 and F.flashdp_checkpoint8_bytes(4, -1) == 0
    assert F.flashdp_checkpoint8_bytes(1 << 22, 1 << 16) == (1 << 38) + (1 << 33)                  # past 32 bits
    for B, T, d in ((1, 1, 1), (8, 2048, 5120), (256, 1, 512), (3, 77, 12345), (1 << 19, 1, 8)):
        for dt in (F.BF16, F.F16, F.F32):
            # at least one partial sum per sample, and not a share of the activations that matters
            for n, got in ((d, F.flashdp_activation_workspace_bytes(B, T, d, dt)), (2 * d, F.flashdp_layernorm_workspace_bytes(B, T, d, dt)),
                           (d, F.flashdp_layernorm_workspace_bytes(B, T, d, dt, False))):
                assert 4 * B * n + 4 * B <= got <= 4 * B * n * (3 + T / 16) + 16 * B * (n // 64 + 1) + 2048, (B, T, d, got)
    assert F.flashdp_activation_workspace_bytes(0, 1, 8, 0) == 0 and F.flashdp_layernorm_workspace_bytes(1, 1, 8, 3) == 0
    mk = lambda p, d: dict(X=None, dY=None, d_in=p, d_out=d, C=1.0, sigma=1.0, seed=0, layer=0, out_grad=None)   # noqa: E731
    L = [mk(96, 40), mk(200, 16)]
    for s in ("twopass", "scratch", "overlap"):
        assert F.flashdp_workspace_bytes_checkpoint8(L, 3, 5, F.BF16, s) == F.flashdp_workspace_bytes(L, 3, 5, F.BF16, s) + 6144      # 3 * 5 * 200 * 2, up to 256
    assert F.flashdp_workspace_bytes_checkpoint8([mk(0, 8)], 3, 5, F.BF16, "scratch") == 0


def test_the_python_layer_refuses_what_is_no_such_buffer():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(F.FlashDPError) as e:          # host memory
        F.flashdp_linear_forward(x, x, None, None, 4, 8, 4, F.BF16, None, x)
    assert e.value.status == INV
    for t in (x, None):
        with pytest.raises((F.FlashDPError, AttributeError)):
            F.flashdp_checkpoint8_pack(t, 4, 8, F.BF16, torch.zeros(64, dtype=torch.uint8))
    with pytest.raises(F.FlashDPError):
        F.activation_code("swish")
    from paper_2507_01154_amd.autograd import DPLinear
    with pytest.raises(ValueError):
        DPLinear(8, 8, device="cpu", checkpoint="4bit")
    with pytest.raises(F.FlashDPError):
        DPLinear(8, 8, device="cpu", activation="tanh")


def test_new_entry_points_are_plain_c_and_link(tmp_path):
    names = ("flashdp_linear_forward", "flashdp_activation_dp_grad", "flashdp_activation_workspace_bytes", "flashdp_layernorm_forward",
             "flashdp_layernorm_dp_grad", "flashdp_layernorm_workspace_bytes", "flashdp_checkpoint8_bytes", "flashdp_checkpoint8_pack",
             "flashdp_checkpoint8_unpack", "flashdp_block_dp_grad_checkpoint8", "flashdp_workspace_bytes_checkpoint8")
    src = tmp_path / "check.c"
    src.write_text('#include <stdio.h>\n#include "flashdp.h"\ntypedef void (*fn_t)(void);\nint main(void) {\n  fn_t syms[] = {%s};\n'
                   '  printf("%%zu\\n", sizeof(syms) / sizeof(syms[0]));\n  return flashdp_checkpoint8_bytes(2, 64) == 132 ? 0 : 1;\n}\n'
                   % ", ".join("(fn_t)" + n for n in names))
    exe, lib_dir = str(tmp_path / "check"), os.path.join(ROOT, "paper_2507_01154_amd")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I" + os.path.join(ROOT, "include"), "-o", exe, str(src), "-L" + lib_dir, "-lflashdp",
                           "-Wl,-rpath," + lib_dir])
    assert subprocess.run([exe], capture_output=True, text=True).stdout.split() == [str(len(names))]


def test_no_kernel_of_the_layers_spills_registers(tmp_path):
    from paper_2507_01154_amd import build as Bd
    res = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature",
                          "-Xclang", "-packed-fp32-ops", "--cuda-device-only", "-c", "-Rpass-analysis=kernel-resource-usage", Bd.sources()[1],
                          "-o", str(tmp_path / "layers.o")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    kernels, cur = {}, None
    for line in res.stderr.splitlines():
        m = re.search(r"Function Name: (\S+)", line)
        if m:
            cur = m.group(1)
        m = re.search(r"remark:.*(VGPRs Spill|ScratchSize \[bytes/lane\]): (\d+)", line)
        if m and cur:
            kernels.setdefault(cur, {})[m.group(1)] = int(m.group(2))
    assert len(kernels) > 40
    for k, u in kernels.items():
        assert u.get("VGPRs Spill", 0) == 0 and u.get("ScratchSize [bytes/lane]", 0) == 0, (k, u)


def test_sizes_whose_bytes_pass_64_bits_are_refused():
    rows, d = 1 << 39, 1 << 25                            # 2^64 elements
    for name, good, change in (("flashdp_linear_forward", FORWARD, dict(rows=rows, d_in=d)), ("flashdp_linear_forward", FORWARD, dict(rows=rows, d_out=d)),
                               ("flashdp_layernorm_forward", NORM, dict(rows=rows, d=d)), ("flashdp_activation_dp_grad", ACTIVATION, dict(B=1 << 9, T=1 << 30, d=d)),
                               ("flashdp_layernorm_dp_grad", NORM_GRAD, dict(B=1 << 9, T=1 << 30, d=d)),
                               ("flashdp_checkpoint8_pack", dict(a=A, rows=4, d=8, dtype=0, b=B_, stream=None), dict(rows=rows, d=d))):
        refused(name, good, change, SHAPE)
    assert F.flashdp_checkpoint8_bytes(rows, d) == 0 and F.flashdp_checkpoint8_bytes(1 << 33, 1 << 25) == (1 << 58) + (1 << 53)
    assert F.flashdp_activation_workspace_bytes(1 << 9, 1 << 30, d, 0) == 0 and F.flashdp_layernorm_workspace_bytes(1 << 9, 1 << 30, d, 0) == 0


def test_buffers_of_a_call_are_on_one_device():
    from paper_2507_01154_amd import binding

    class Elsewhere:      # a tensor as the checks see it, on device 1
        dtype, shape, device = torch.float32, (8,), "cuda:1"
        get_device, numel, is_contiguous, data_ptr, element_size = (lambda s: 1), (lambda s: 8), (lambda s: True), (lambda s: A), (lambda s: 4)

    assert binding._buffer(Elsewhere(), 8, torch.float32, "x", 1) == A and binding._room(Elsewhere(), "x", 1) == (A, 32) and binding._room(None, "x", 0) == (None, 0)
    for bad in (lambda: binding._buffer(Elsewhere(), 8, torch.float32, "x", 0), lambda: binding._room(Elsewhere(), "x", 0),
                lambda: binding._room(torch.zeros(64), "x", 0), lambda: binding._buffer(Elsewhere(), 9, torch.float32, "x", 1)):
        with pytest.raises(F.FlashDPError) as e:
            bad()
        assert e.value.status == INV


def test_modules_refuse_inputs_of_other_shapes():
    from paper_2507_01154_amd.autograd import DPLayerNorm, DPLinear
    lin, ln = DPLinear(8, 8, device="cpu", bias=True, dtype=torch.float32), DPLayerNorm(8, device="cpu", dtype=torch.float32)
    for shape in ((2, 4, 4), (2, 16), (8,), (64,)):       # 2 x 4 x 4: as many elements as four rows of 8
        for m in (lin, ln):
            with pytest.raises(TypeError):
                m(torch.zeros(shape))
    for residual in (torch.zeros(2, 1, 8), torch.zeros(2, 3, 8, dtype=torch.float64), torch.zeros(6, 8)):
        with pytest.raises(TypeError):
            lin(torch.zeros(2, 3, 8), residual=residual)
