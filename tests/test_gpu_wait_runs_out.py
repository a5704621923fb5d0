"""A wait inside a kernel of the training operators that runs out: the kernel returns, the whole warp is told the same, and status reports it once."""
import pytest
import torch

from paper_1903_04488_b200 import ssgd as S
from paper_1903_04488_b200 import train_ops as T


def test_the_hook_refuses_limits_that_are_none():
    lib = S.lib()
    for limit, told in ((0, 4096), (999, 4096), (1000000001, 4096), (1000, None)):
        assert lib.ssgd_test_run_out(limit, told, None) == S.EINVAL
    assert lib.ssgd_test_run_out(1000, 4098, None) == S.EALIGN


@pytest.mark.gpu
def test_a_wait_that_runs_out_is_reported_and_every_lane_is_told_the_same(cuda_device):
    lib = S.lib()
    told = torch.full((32,), 7, dtype=torch.int32, device="cuda")
    T.status()
    # half of the lanes give up after 0.2 ms, the barrier completes for the others: the warp goes one way all the same
    assert lib.ssgd_test_run_out(200_000, told.data_ptr(), torch.cuda.current_stream().cuda_stream) == S.OK
    with pytest.raises(S.SsgdError) as e:
        T.status()
    assert e.value.code == S.EDEVICE
    T.status()                                 # reported once
    assert told.tolist() == [0] * 32
    x = torch.randn(300, 200, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    assert T.orthogonalize(x).isfinite().all()
    T.status()
