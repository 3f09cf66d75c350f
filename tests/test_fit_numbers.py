"""Numbers that the fields of the C structures do not hold are refused, not cut to their low bits."""
import pytest
import torch

from paper_2206_05279_amd import binding as pb

OVER = [(1 << 32) + 5, 1 << 32, -1]


@pytest.mark.parametrize("n", OVER)
def test_sizes_of_workspaces(n):
    for call in (lambda: pb.pilc_logprobs_workspace_size(n, 4), lambda: pb.pilc_logprobs_workspace_size(4, n),
                 lambda: pb.pilc_logprobs_workspace_size(4, 4, n), lambda: pb.pilc_norm_workspace_size(n, 8),
                 lambda: pb.pilc_norm_workspace_size(8, n)):
        with pytest.raises(pb.PilcError) as e:
            call()
        assert e.value.code == pb.PILC_E_ARG


def test_the_most_rows_are_no_error():
    assert pb.pilc_logprobs_workspace_size((1 << 32) - 1, 4) >= 256 and pb.pilc_norm_workspace_size((1 << 32) - 1, 8) >= 256


@pytest.mark.gpu
def test_tensors_of_more_rows_than_are_counted():
    rows = (1 << 32) + 5
    x, y = (torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    some = torch.empty(5, dtype=torch.float32, device="cuda:0")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda:0")
    for call in (lambda: pb.pilc_norm_forward(x, None, None, y), lambda: pb.pilc_logprobs(x, None, entropy=some, workspace=ws)):
        with pytest.raises(pb.PilcError) as e:
            call()
        assert e.value.code == pb.PILC_E_ARG
    del x, y
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("step", [-1, 0, 1 << 64])
def test_steps_that_are_none(step):
    p, g, m, v = (torch.zeros(8, device="cuda:0") for _ in range(4))
    tensors = pb.make_adamw_tensors([p], [g], [m], [v])
    with pytest.raises(pb.PilcError) as e:
        pb.pilc_adamw_step(tensors, 1e-3, 0.9, 0.999, 1e-8, step)
    assert e.value.code == pb.PILC_E_ARG
