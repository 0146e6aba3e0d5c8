"""Calls around the weight gradient that the other files do not make: noise inside a capture, schedules of several layers on
checkpoints, sums over many samples, single products, rows that decide a result alone."""
import pytest
import torch

import paper_2507_01154_amd as F
from gpu_util import DEV, env

pytestmark = pytest.mark.gpu


def test_a_module_that_counts_its_steps_does_not_have_its_noise_captured():
    from paper_2507_01154_amd.autograd import DPLinear
    make = lambda **kw: DPLinear(64, 48, C=1.0, bias=True, schedule="twopass", device=DEV, **kw)     # noqa: E731
    refused, quiet = make(sigma=0.5), make(sigma=0.0)
    x, dy, total = torch.randn(2, 9, 64, device=DEV).bfloat16(), torch.randn(2, 9, 48, device=DEV).bfloat16(), torch.zeros(1, device=DEV)
    warm = make(sigma=0.0)               # (kernels are launched eagerly once, by a module that is not captured)
    want = [t.clone() for t in torch.autograd.grad(warm(x), list(warm.parameters()), dy)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(RuntimeError, match="replay"):
            torch.autograd.grad(refused(x), list(refused.parameters()), dy)
        got = torch.autograd.grad(quiet(x), list(quiet.parameters()), dy)
        total.add_(1.0)                  # the capture goes on
    for rep in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert float(total) == rep + 1 and all(torch.equal(a, b) for a, b in zip(got, want))


def packed_and_back(x, rows, d, code):
    p, y = torch.empty(F.flashdp_checkpoint8_bytes(rows, d), dtype=torch.uint8, device=DEV), torch.empty_like(x)
    F.flashdp_checkpoint8_pack(x, rows, d, code, p)
    F.flashdp_checkpoint8_unpack(p, rows, d, code, y)
    return p, y


def gradients(call, X, dYs, B, T, P, code, schedule, workspace=None):
    layers = [dict(X=X, dY=dY, d_in=P, d_out=dY.shape[-1], C=1.0 + k, sigma=0.5, seed=7, layer=k, out_grad=torch.empty(dY.shape[-1], P, device=DEV),
                   out_norms=torch.empty(B, device=DEV)) for k, dY in enumerate(dYs)]
    call(layers, B, T, code, schedule, workspace)
    torch.cuda.synchronize()
    return [t for L in layers for t in (L["out_grad"], L["out_norms"])], F.flashdp_last_schedule()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,T,P,Ds", [(8, 256, 2048, (2048, 1024, 2048)), (4, 16, 256, (256, 512)), (6, 1, 264, (512, 96)), (3, 200, 100, (33, 65)), (16, 64, 64, (64,) * 18)])
@pytest.mark.parametrize("schedule", ["auto", "overlap", "scratch", "twopass"])
def test_layers_on_one_checkpoint_take_the_schedule_that_they_take_on_the_unpacked_activation(schedule, B, T, P, Ds, dtype):
    """With the library's memory, and with the caller's: the same schedule, and the same bits."""
    torch.manual_seed(T)
    x, dYs = torch.randn(B * T, P, device=DEV).to(dtype), [torch.randn(B, T, d, device=DEV).to(dtype) for d in Ds]
    code = F.dtype_code(x)
    p, y = packed_and_back(x, B * T, P, code)
    room = (B * T * P * x.element_size() + 255) // 256 * 256
    run = dYs[:16]           # (of 18 layers two go to a call of their own)
    for nbytes in (None, F.flashdp_workspace_bytes([dict(X=None, dY=None, d_in=P, d_out=d, C=1.0, sigma=0.0, seed=0, layer=0, out_grad=None) for d in Ds], B, T, code, schedule)):
        ws = lambda n: None if nbytes is None else torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)       # noqa: E731
        got, how = gradients(F.flashdp_block_dp_grad_checkpoint8, p, dYs, B, T, P, code, schedule, ws((nbytes or 0) + room))
        want, by_hand = gradients(F.flashdp_block_dp_grad_micro, y, run, B, T, P, code, schedule, ws(nbytes or 0))
        assert (how == by_hand or len(Ds) > 16) and all(torch.equal(a, b) for a, b in zip(got, want)), (nbytes, how, by_hand)


def test_the_schedule_that_replaces_the_argument_has_its_workspace():
    x, dYs = torch.randn(8 * 64, 512, device=DEV).bfloat16(), [torch.randn(8, 64, 256, device=DEV).bfloat16()]
    p, y = packed_and_back(x, 8 * 64, 512, F.BF16)
    want, _ = gradients(F.flashdp_block_dp_grad_micro, y, dYs, 8, 64, 512, F.BF16, "scratch")
    with env(FLASHDP_SCHEDULE="scratch"):
        got, how = gradients(F.flashdp_block_dp_grad_checkpoint8, p, dYs, 8, 64, 512, F.BF16, "twopass")
    assert how == "scratch" and all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_overlapped_schedule_is_taken_from_checkpoints_as_it_is_without_them():
    B, T, P = 4, 1024, 4096
    x, dYs = torch.randn(B * T, P, device=DEV).bfloat16(), [torch.randn(B, T, P, device=DEV).bfloat16() for _ in range(2)]
    p, y = packed_and_back(x, B * T, P, F.BF16)
    want, by_hand = gradients(F.flashdp_block_dp_grad_micro, y, dYs, B, T, P, F.BF16, "auto")
    got, how = gradients(F.flashdp_block_dp_grad_checkpoint8, p, dYs, B, T, P, F.BF16, "auto")
    assert by_hand == how == "overlap" and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T", [1, 40])
@pytest.mark.parametrize("deferred", [False, True])
def test_captured_layers_without_an_epilogue_outlive_the_librarys_workspace(deferred, T):
    """Replayed beside eager calls that make the library's workspace grow, and after it was given back.  The captured modules are never run eagerly."""
    from contextlib import nullcontext
    from paper_2507_01154_amd.autograd import DPLinear, deferred_weight_grads
    torch.manual_seed(2)
    eager, captured = ([DPLinear(64, 96, C=1.0, sigma=0.5, seed=3, layer=k, device=DEV, auto_step=False) for k in range(3)] for _ in range(2))
    for a, b in zip(eager, captured):
        a.load_state_dict(b.state_dict())
    x, dy = torch.empty(3, T, 64, device=DEV, dtype=torch.bfloat16), torch.empty(3, T, 96, device=DEV, dtype=torch.bfloat16)

    def step(ms):
        for m in ms:
            m.weight.grad = None
        with deferred_weight_grads() if deferred else nullcontext():
            for m in ms:
                m(x).backward(dy)
        return [m.weight.grad for m in ms]

    def draw(seed):
        torch.manual_seed(seed)
        x.normal_()
        dy.normal_()

    draw(1)
    step(eager)
    torch.cuda.synchronize()
    F.flashdp_release()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(captured)
    for rep in range(3):
        draw(rep)
        want = [t.clone() for t in step(eager)]
        big = 256 << rep
        a, o = torch.ones(2, 64, big, device=DEV, dtype=torch.bfloat16), torch.empty(big, big, device=DEV)
        F.flashdp_block_dp_grad([dict(X=a, dY=a, d_in=big, d_out=big, C=1.0, sigma=0.0, seed=0, layer=0, out_grad=o)], 2, 64, F.BF16, "scratch")
        if rep == 2:
            F.flashdp_release()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert float((g.float() - w.float()).norm() / w.float().norm()) <= 2.0 ** -8, rep      # (one step of bfloat16 where the order of additions differs)


@pytest.mark.parametrize("B", [300, 5000, 1 << 18])
@pytest.mark.parametrize("n", [1, 40])
def test_sums_over_many_equal_samples_keep_their_bits(B, n):
    """Nothing clips, so the factors are 1 and the sum is B times a number whose roundings on the way all point one way.  Added up in 64 bits and
    rounded once: off by half a step of fp32, 2^-24, and less than another for the 64 bits."""
    g = torch.full((B, 1, n), 1.0 / 3.0, device=DEV) * torch.linspace(1, 2, n, device=DEV)
    out = torch.empty(n, device=DEV)
    F.flashdp_activation_dp_grad(g, None, False, B, 1, n, F.F32, None, 1e6, 0.0, 0, 0, None, out)
    want = B * g[0, 0].cpu().double()
    assert bool(((out.cpu().double() - want).abs() <= 1.01 * 2.0 ** -24 * want).all()), float(((out.cpu().double() - want).abs() / want).max() * 2 ** 24)
    F.flashdp_activation_dp_grad(g, None, False, B, 1, n, F.F32, None, 1e6, 0.0, 0, 0, None, out, accumulate=True)
    assert bool(((out.cpu().double() - 2 * want).abs() <= 2.02 * 2.0 ** -24 * 2 * want).all())


@pytest.mark.parametrize("kernel", [None, 10, 11])
@pytest.mark.parametrize("K", [64, 128, 773, 4096])
@pytest.mark.parametrize("kind", ["just above one", "one product", "rectified", "normal"])
def test_single_precision_products_keep_single_precision(kind, K, kernel):
    """fp32 operands in bfloat16 parts, where they are taken.  u = 2^-24.  A product of two floats: the parts left out are below 2^-22 of it, 4 u.  A k-tile of 32
    products: six matrix instructions, of which the last, with the largest parts, cuts its sum off within a step, 2 u, and the ones before it, of
    parts below 2^-7, less than that together.  Then K / 32 additions that round by u each.  Products of one sign show whether what is cut off adds up."""
    rows, D = 200, 264
    g = torch.Generator().manual_seed(K)
    if kind == "just above one":
        x, w = (1 + torch.rand(n, K, generator=g) * 2.0 ** -6 for n in (rows, D))
    elif kind == "one product":
        x, w = torch.zeros(rows, K), 1 + torch.rand(D, K, generator=g)
        x[torch.arange(rows), torch.randint(K, (rows,), generator=g)] = 1 + torch.rand(rows, generator=g)
        x[0, x[0] != 0] = 1 + 2.0 ** -7 - 2.0 ** -23
        w[0] = 1 + 2.0 ** -7 - 2.0 ** -23
    elif kind == "rectified":
        x, w = torch.randn(rows, K, generator=g).clamp(min=0), torch.rand(D, K, generator=g)
    else:
        x, w = torch.randn(rows, K, generator=g), torch.randn(D, K, generator=g)
    y = torch.empty(rows, D, device=DEV)
    with env(FLASHDP_FORWARD=kernel):
        F.flashdp_linear_forward(x.to(DEV), w.to(DEV), None, None, rows, K, D, F.F32, None, y)
        assert kernel is None or F.flashdp_last_kernel() == "forward_split_kernel"
    x64, w64 = x.double(), w.double()
    want, size = x64 @ w64.T, x64.abs() @ w64.abs().T
    u = 2.0 ** -24
    # (the fp32 instructions, where the parts are not taken, add K products in a row)
    steps = 4 + 2 + 2 + (K + 31) // 32 if kernel is not None else K + 2
    assert bool(((y.cpu().double() - want).abs() <= steps * u * size).all()), float(((y.cpu().double() - want).abs() / size).max() / u)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 6])
@pytest.mark.parametrize("d", [72, 75, 1032, 1035, 8200, 16408, 20001])
def test_a_mean_whose_product_with_rstd_overflows(d, T, dtype):
    """Constant rows: x - mean is zero, and so is every normalised value, but mean * rstd is not finite: what lies between a row's end and the last
    thread's must not enter its sums as zero times infinity.  dx = rstd (a - mean(a)): d / 64 + 10 additions of fp32 and one rounding to the type."""
    B, c, r = 2, 2.0 ** 121, 2.0 ** 8
    torch.manual_seed(d)
    x, dy = torch.full((B * T, d), c, device=DEV, dtype=dtype), torch.randn(B, T, d, device=DEV).to(dtype)
    gam = torch.randn(d, device=DEV).to(dtype)
    mean, rstd = torch.full((B * T,), c, device=DEV), torch.full((B * T,), r, device=DEV)
    dx, g, n = torch.empty_like(dy), torch.empty(2, d, device=DEV), torch.empty(B, device=DEV)
    F.flashdp_layernorm_dp_grad(x, dy, gam, mean, rstd, B, T, d, F.dtype_code(x), 1e6, 0.0, 0, 0, dx, g, n)
    dy64, a = dy.cpu().double(), dy.cpu().double() * gam.cpu().double()
    want = r * (a - a.mean(-1, keepdim=True))
    slack = r * ((d / 64 + 10) * 2.0 ** -24 * a.abs().mean(-1, keepdim=True) + 2.0 ** -22 * a.abs())
    assert bool(((dx.cpu().double() - want).abs() <= 1.01 * slack + torch.finfo(dtype).eps / 2 * want.abs()).all())
    total = dy64.sum(1)
    assert bool((g[0] == 0).all()) and bool(((g[1].cpu().double() - total.sum(0)).abs() <= (B * T + 4) * 2.0 ** -24 * dy64.abs().sum((0, 1))).all())
    assert bool(((n.cpu().double() - total.norm(dim=1)).abs() <= (T + 4) * 2.0 ** -24 * dy64.abs().sum(1).norm(dim=1)).all())


# rows of 2048 elements on both sides of 2^30 and 2^31 elements, the ends of both samples, and some others; each with a power of two of its own
MARKED = [0, 1, 255, 256, 4095, 99999, 524287, 524288, 549999, 550000, 550001, 786432, 1000003, 1048575, 1048576, 1048577, 1099990, 1099999]


def marked_gradient(B, rows, d):
    """dY that is zero but for the marked rows, and its sum over each sample's tokens: every row read once or the sum is another number, exactly."""
    dy, per = torch.zeros(rows, d, device=DEV, dtype=torch.bfloat16), 1.0 + torch.arange(d, device=DEV) % 3
    sums = torch.zeros(B, d, dtype=torch.float64, device=DEV)
    for k, r in enumerate(MARKED):
        dy[r] = (2.0 ** k * per).bfloat16()
        sums[r * B // rows] += 2.0 ** k * per.double()
    return dy, sums


def test_every_row_of_long_inputs_enters_the_gradients_of_vectors_once():
    """1100000 x 2048: bias (ReLU of ones, Z as it is and in 8 bits) and layer norm (mean 0, rstd 1, x of -2 .. 2).  All sums are whole numbers below 2^24."""
    B, rows, d = 2, 1100000, 2048
    T = rows // B
    dy, sums = marked_gradient(B, rows, d)
    z = torch.ones(rows, d, device=DEV, dtype=torch.bfloat16)
    z8 = torch.empty(F.flashdp_checkpoint8_bytes(rows, d), dtype=torch.uint8, device=DEV)
    F.flashdp_checkpoint8_pack(z, rows, d, F.BF16, z8)
    g, n = torch.empty(d, device=DEV), torch.empty(B, device=DEV)
    for kept, eight in ((z, False), (z8, True)):
        F.flashdp_activation_dp_grad(dy, kept, eight, B, T, d, F.BF16, "relu", 1e30, 0.0, 0, 0, None, g, n)
        assert torch.equal(g.double(), sums.sum(0))
        assert bool(((n.double() - sums.norm(dim=1)).abs() <= 2.0 ** -24 * sums.norm(dim=1)).all())
    del z8
    x = z
    x.copy_(((torch.arange(rows, device=DEV)[:, None] * 7 + torch.arange(d, device=DEV) * 3) % 5 - 2).to(torch.bfloat16))
    want = torch.zeros(B, 2, d, dtype=torch.float64, device=DEV)
    for r in MARKED:
        want[r * B // rows, 0] += dy[r].double() * x[r].double()
    want[:, 1] = sums
    gn, mean, rstd = torch.empty(2, d, device=DEV), torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
    F.flashdp_layernorm_dp_grad(x, dy, torch.ones(d, device=DEV, dtype=torch.bfloat16), mean, rstd, B, T, d, F.BF16, 1e30, 0.0, 0, 0, None, gn, n)
    assert torch.equal(gn.double(), want.sum(0))
    norms = want.reshape(B, -1).norm(dim=1)
    assert bool(((n.double() - norms).abs() <= 2.0 ** -24 * norms).all())


@pytest.mark.parametrize("rows,K,D,dtype,kernel", [(1, 4097, 1000, "bf16", "forward_rows_kernel"), (64, 2049, 1000, "f16", "forward_tile_kernel"), (8, 769, 50257, "f16", "forward_tile_kernel"),
                                                   (8, 770, 8192, "bf16", "forward_rows_kernel"), (33, 515, 50257, "fp32", "forward_split_kernel"), (16, 515, 4000, "fp32", "forward_rows_kernel"),
                                                   (64, 33, 20001, "bf16", "forward_tile_kernel"), (64, 3001, 17001, "bf16", "forward_tile_kernel"), (2, 33, 50257, "fp32", "forward_tile_kernel")])
def test_few_rows_that_no_chunks_divide_take_the_kernel_of_the_shorter_rounds(rows, K, D, dtype, kernel):
    from test_gpu_layers import check_forward
    check_forward(rows, K, D, dtype, "gelu_tanh", True, False, "8bit" if dtype != "fp32" else "dtype", seed=K)
    check_forward(rows, K, D, dtype, "none", False, True, None, seed=D)
    assert F.flashdp_last_kernel() == kernel
