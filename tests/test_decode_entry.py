"""Host side of the decoder operators on PyTorch tensors: refusals that need no GPU."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def pb():
    from paper_1712_01084_b200 import binding
    return binding


def test_norm_refuses_host_tensors(pb):
    with pytest.raises(ValueError, match="x must be a CUDA tensor"):
        pb.pp_rmsnorm_q8(torch.zeros(2, 8), torch.ones(8))
    with pytest.raises(ValueError):
        pb.pp_rmsnorm_q8(torch.zeros(()), torch.ones(8))
    with pytest.raises(ValueError):
        pb.pp_rmsnorm_q8(torch.zeros(2, 2, 8), torch.ones(8))


def test_norm_refuses_what_is_no_tensor(pb):
    with pytest.raises(TypeError, match="x must be a tensor"):
        pb.pp_rmsnorm_q8([1.0, 2.0], torch.ones(2))
    with pytest.raises(TypeError, match="weight must be a tensor"):
        pb.pp_rmsnorm_q8(torch.zeros(2, 8), None)


class _Closed:
    """A layer whose handle is gone, as close() leaves it."""
    M = N = H = 8
    top_k, device = 1, 0

    class _h:
        value = None


def test_layers_refuse_host_tensors(pb):
    pb._load_torch()
    with pytest.raises(ValueError, match="on device 0"):
        pb.pp_q4_forward(_Closed, torch.zeros(1, 8))
    with pytest.raises(ValueError, match="on device 0"):
        pb.pp_moe_forward(_Closed, torch.zeros(1, 8))
    with pytest.raises(TypeError):
        pb.pp_q4_forward(_Closed, None)
    with pytest.raises(TypeError):
        pb._fast.q4_forward(1, 2, 3)
