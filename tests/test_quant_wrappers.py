"""What the 8-bit wrappers allocate, refuse and launch, and where: host checks, nothing runs
on a GPU.  Launches and allocations are recorded in place of being made."""
import pytest


class Stream:
    """What a call asks a stream for."""

    def __init__(self, index=0):
        import torch
        self.device = torch.device("cuda", index)
        self.cuda_stream = 0x5000 + index


@pytest.fixture
def quant(monkeypatch):
    """The module with launches recorded: (device, stream, arguments)."""
    from paper_2606_15615_amd import quant as m
    m.launches = []
    monkeypatch.setattr(m, "_launch",
                        lambda fn, device, stream, *a: m.launches.append((device, stream, a)))
    yield m
    del m.launches


def test_scales_of_a_matrix_are_not_filled(quant, monkeypatch):
    """A fill would run on the current stream and the kernel that writes the scales on
    the call's, in no order."""
    import torch

    def no_fill(*a, **k):
        raise AssertionError("a fill on the current stream")
    for name in ("zeros", "full", "ones"):
        monkeypatch.setattr(torch, name, no_fill)
    for shape in ((70, 200), (3, 130, 260)):
        m = quant.quantize_matrix(torch.empty(shape), stream=Stream())
        assert m.q.shape[:-2] == shape[:-2] and (m.N, m.K) == shape[-2:]
    assert len(quant.launches) == 2


def test_new_tensors_belong_to_the_calls_stream(quant, monkeypatch):
    import torch
    now, made, empty = [None], [], torch.empty

    class on:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            now[0] = self.stream

        def __exit__(self, *a):
            now[0] = None

    def recorded(*a, **k):
        made.append(now[0])
        return empty(*a, **k)

    r = quant.QuantRows(6, 200, device="cpu")
    W = quant.quantize_matrix(torch.empty(70, 200))
    ws = quant.linear_workspace(5, 200, "cpu")
    x, out = torch.empty(5, 200), torch.empty(5, 70)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", recorded)
    s = Stream()
    for call, n in ((lambda **k: r.read(**k), 1), (lambda **k: quant.quantize_matrix(x, **k), 2),
                    (lambda **k: quant.linear(x, W, workspace=ws, **k), 1),
                    (lambda **k: quant.linear(x, W, out=out, workspace=ws, **k), 0)):
        for stream in (None, s):
            made.clear()
            call(stream=stream)
            assert made == [stream] * n and quant.launches[-1][1] is stream


def test_a_stream_of_another_device_is_refused():
    import torch
    from paper_2606_15615_amd import quant

    def never(*a):
        raise AssertionError("launched")
    with pytest.raises(ValueError, match="stream is one of cuda:1"):
        quant._launch(never, torch.device("cuda", 0), Stream(1))


def test_a_product_in_place_is_refused(quant):
    """Blocks of a product read rows of x while others write rows of out."""
    import torch
    W = quant.quantize_matrix(torch.empty(200, 200))
    x = torch.empty(3, 200)
    n = len(quant.launches)
    with pytest.raises(ValueError, match="out is x"):
        quant.linear(x, W, out=x)
    assert len(quant.launches) == n
    wide = torch.empty(3, 400)                     # halves of the same rows are apart
    quant.linear(wide[:, :200], W, out=wide[:, 200:])
    assert quant.linear(x[:0], W, out=x[:0]).shape == (0, 200)
