"""Calls of the operators for drafted tokens, and of sampling, that the host refuses; nothing is launched, so no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2410_23668_b200 import binding as kl, build

OK, BAD, SHAPE = kl.KL_OK, kl.KL_ERR_INVALID_ARG, kl.KL_ERR_UNSUPPORTED_SHAPE
P = 4096   # stands for a device pointer; a refused call never follows it


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return kl.lib()


def sample_call(lib, x=P, stride=1000, n=3, vocab=1000, u=P, tokens=P):
    return lib.kl_sample(x, stride, n, vocab, u, None, None, None, None, tokens, None, None, None)


def test_sample(lib):
    for over in (dict(x=None), dict(u=None), dict(tokens=None), dict(vocab=0), dict(stride=999), dict(stride=-1000), dict(stride=1 << 40)):
        assert sample_call(lib, **over) == BAD, over
    for over in (dict(vocab=327681, stride=327681), dict(n=(1 << 24) + 1)):
        assert sample_call(lib, **over) == SHAPE, over
    assert sample_call(lib, n=0, x=None) == OK


def test_sample_binding():
    x, u, t = torch.zeros(2, 8), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(kl.KlError):   # not on a CUDA device
        kl.kl_sample(x, u, t)
