"""Sizes that a 32-bit argument cannot hold are refused, not cut to their lowest 32 bits (no GPU needed)."""
import pytest
import torch

import paper_2304_14698_b200 as xrl

MANY = 2 ** 32 + 5


@pytest.fixture(scope="module", autouse=True)
def library():
    from paper_2304_14698_b200 import build
    build.build()


def one(*shape):
    return torch.zeros(1).expand(*shape)


@pytest.mark.parametrize("call", [
    lambda: xrl.xrl_logprob(one(MANY, 1)), lambda: xrl.xrl_logprob(one(1, MANY)), lambda: xrl.xrl_logprob(one(2, 7), top=MANY),
    lambda: xrl.xrl_logprob_grad(one(MANY, 1), one(MANY, 2)), lambda: xrl.xrl_logprob_grad(one(1, MANY), one(1, 2)),
    lambda: xrl.xrl_orthogonalise(one(MANY, 1)), lambda: xrl.xrl_orthogonalise(one(1, MANY)), lambda: xrl.xrl_orthogonalise(one(MANY, 2, 2)),
    lambda: xrl.xrl_orthogonalise_workspace(0, MANY, 2, 2), lambda: xrl.xrl_orthogonalise_workspace(0, 1, MANY, 2),
    lambda: xrl.xrl_orthogonalise_workspace(0, 1, 2, MANY)])
def test_refused(call):
    with pytest.raises(xrl.XrlError) as e:
        call()
    assert e.value.status == 8


def test_layers_of_a_blob_that_is_none():
    """A view that skips entries, one whose storage goes on behind it, and a table."""
    m = dict(T=13, S=8, H=64, K=2, L=3, Hm=32, Dg=1, dtype="fp32", A_max=8)
    size = (2 * 8 + 13) * 64 + 64 + 3 * (64 * 64 + 3 * 64)
    assert xrl.layer_matrices(m, torch.zeros(size)).shape == (3, 64, 64)
    for bad in (torch.zeros(2 * size)[::2], torch.zeros(2 * size)[:size - 1], torch.zeros(1, size), torch.zeros(size - 1)):
        with pytest.raises(xrl.XrlError) as e:
            xrl.layer_matrices(m, bad)
        assert e.value.status == 1
    for bad in (torch.zeros(2 * size)[::2], torch.zeros(2 * size)[:size - 1]):
        with pytest.raises(xrl.XrlError):
            xrl.orthogonalise_layers(m, bad)


@pytest.mark.parametrize("steps", [0, -1, 65, MANY, 5 - 2 ** 32])
def test_steps(steps):
    with pytest.raises(xrl.XrlError) as e:
        xrl.xrl_orthogonalise(one(4, 4), steps=steps)
    assert e.value.status == 1 and "steps" in str(e.value)
