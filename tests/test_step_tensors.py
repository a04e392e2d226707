"""Tensors that the calls around attention and the gradients refuse before anything is launched, without a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def lx():
    from paper_2510_15964_amd import build
    build.ensure()
    from paper_2510_15964_amd import lx
    return lx


def test_a_rotary_table_on_the_host_is_refused(lx):
    with pytest.raises(AssertionError):
        lx.lx_rope_table(32, 8, out=torch.empty(8, 32))


def test_gradients_on_the_host_are_refused(lx):
    with pytest.raises(AssertionError):
        lx.GradSet([torch.ones(8)])
