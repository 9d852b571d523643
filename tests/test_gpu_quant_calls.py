"""Calls of the 8-bit operators on other streams, in other forms and at the ends of
their ranges, on the GPU, against the 64-bit oracle (oracle/quant_oracle.py) or the
same call in its usual form."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import quant_oracle as Q


def say(msg):
    print(msg, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_15615_amd import _lib
    _lib.load()


def _busy(t, n=20):
    """Work for the current stream, so that what it is asked for next comes late."""
    for _ in range(n):
        t = t @ t
    return t


@pytest.mark.parametrize("shape", [(300, 700), (2, 130, 260)])
def test_matrix_on_another_stream(shape):
    """While the current stream is busy: the bytes of the call on the current one."""
    import torch
    from paper_2606_15615_amd import quant
    say(f"  matrix {shape} on a stream of its own")
    g = torch.Generator(device="cuda:0")
    g.manual_seed(3)
    w = torch.randn(*shape, generator=g, device="cuda:0")
    big = torch.randn(2048, 2048, generator=g, device="cuda:0") / 45
    want, nb = quant.quantize_matrix(w), -(-shape[-1] // 128)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        _busy(big)
        got = quant.quantize_matrix(w, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got.q, want.q)
        assert torch.equal(got.scale[..., :nb], want.scale[..., :nb])
