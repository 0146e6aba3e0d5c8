"""The layers around the weight gradient, checked without a device: which schedule a call from checkpoints is sized and refused for."""
import pytest

import paper_2507_01154_amd as F
from gpu_util import env

A, B_, C_ = 0x10000, 0x20000, 0x30000      # fake, aligned, never dereferenced


def layers(*sizes):
    arr = (F.flashdp_layer_t * len(sizes))()
    for k, (p, d) in enumerate(sizes):
        for name, v in dict(X=A + 64 * k, dY=B_, d_in=p, d_out=d, C=1.0, sigma=0.0, seed=0, layer=k, out_grad=C_, out_norms=None).items():
            setattr(arr[k], name, v)
    return arr


def call(arr, B, T, schedule, ws=None, nbytes=0, dtype=F.BF16):
    return F.lib().flashdp_block_dp_grad_checkpoint8(arr, len(arr), B, T, dtype, F.schedule_code(schedule), ws, nbytes, None, 0, 1)


def test_the_schedule_that_replaces_the_argument_is_the_one_a_call_from_checkpoints_is_sized_for():
    arr = layers((1024, 1024), (512, 2048))
    least, parked = (F.flashdp_workspace_bytes_checkpoint8(arr, 8, 100, F.BF16, s) for s in ("twopass", "scratch"))
    assert least < parked
    with env(FLASHDP_SCHEDULE="scratch"):
        assert F.flashdp_workspace_bytes_checkpoint8(arr, 8, 100, F.BF16, "twopass") == parked
        # before anything is enqueued (and before a device is looked for)
        assert call(arr, 8, 100, "twopass", A, least) == F.WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("sizes", [[(8, 8)], [(8, 8), (8, 16)]])
def test_sizes_that_a_schedule_does_not_take_are_refused_before_the_first_layer(sizes):
    """More token blocks than the Gram kernel's grid holds."""
    B, T = 1, 1 << 26
    assert call(layers(*sizes), B, T, "ghost", A, 1 << 60) == F.UNSUPPORTED_SHAPE
    with env(FLASHDP_SCHEDULE="ghost"):
        assert call(layers(*sizes), B, T, "twopass") == F.UNSUPPORTED_SHAPE
