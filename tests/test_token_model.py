"""What the token model refuses before it calls an operator (no GPU needed)."""
import pytest
import torch

from paper_1912_11554_amd.token_model import TokenModel


def _model():
    ids = torch.zeros(3, dtype=torch.int64)
    return TokenModel(None, ids, ids, V=5, D=4, F=6)


def test_trajectories_in_bf16_are_refused():
    m = _model()
    w = m.init(dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="float32"):
        m.sample(w, step_size=0.1, steps=2, num_samples=1)
    with pytest.raises(TypeError, match="float32"):
        m.leapfrog(w, w, w, 0.1, 2)
    mixed = m.init()
    mixed["head"] = mixed["head"].double()
    with pytest.raises(TypeError, match="head"):
        m.sample(mixed, step_size=0.1, steps=2, num_samples=1)


@pytest.mark.parametrize("steps", [0, -1])
def test_trajectories_of_no_steps_are_refused(steps):
    m = _model()
    w = m.init()
    with pytest.raises(ValueError, match="at least one step"):
        m.leapfrog(w, w, w, 0.1, steps)
