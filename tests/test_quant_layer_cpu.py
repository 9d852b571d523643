"""What the layer's wrapper checks of 8-bit weights and caches, on the host: the layer's
memory is the host's, and nothing is launched."""
import pytest


@pytest.fixture
def layer(monkeypatch):
    """Makes a layer whose workspace is host memory, whatever device it is asked for."""
    import torch
    from paper_2606_15615_amd.layer import MoecaLayer
    empty = torch.empty

    def make(d=128, E=4, k=2, d_ff=64, **kw):
        with monkeypatch.context() as m:
            m.setattr(torch, "empty", lambda *a, **ka: empty(*a, **{**ka, "device": "cpu"}))
            return MoecaLayer(d, E, k, d_ff, batch=1, tokens=8, **kw)
    return make


def _bytes(*shape):
    """Zeros at an address that the C calls accept."""
    import torch
    n = 1
    for s in shape:
        n *= s
    t = torch.zeros(n + 256, dtype=torch.uint8)
    at = -t.data_ptr() % 256
    return t[at:at + n].view(*shape)


def _stack(n, N, K):
    from paper_2606_15615_amd import quant
    lib = quant._lib
    return quant.QuantMatrix(_bytes(n, N, lib.moeca_quant_pitch(K)),
                             _bytes(n, -(-N // 128), lib.moeca_quant_scale_pitch(K)), N, K)


def _rows(n, K, norm=False):
    from paper_2606_15615_amd import quant
    lib = quant._lib
    return quant.QuantRows(n, K, q=_bytes(n, lib.moeca_quant_pitch(K)),
                           scale=_bytes(n, lib.moeca_quant_scale_pitch(K)), norm=norm)


@pytest.mark.parametrize("device", ["cuda", "cuda:0"])
def test_the_layers_device_is_its_workspaces(layer, device):
    """"cuda" names the current device; 8-bit weights and caches on it are taken."""
    L = layer(device=device, experts="e4m3", cache="e4m3", n_shared=1)
    assert L.device == L.workspace.device
    w = _bytes(4, 128 * 2)
    L.set_weights_quant(w, None, _stack(4, 64, 128), _stack(4, 128, 64))
    L.set_shared_quant(_stack(1, 64, 128), _stack(1, 128, 64))
    L.bind_attention(w, _rows(8, 128))
    with pytest.raises(ValueError, match="expected 4 quantised matrices"):
        L.set_weights_quant(w, None, _stack(4, 64, 64), _stack(4, 128, 64))


def test_an_attention_cache_with_norms_is_refused(layer):
    """A step would leave its norms those of rows that are gone."""
    L = layer(cache="e4m3")
    x = _bytes(8, 128 * 2)
    with pytest.raises(ValueError, match="without a norm"):
        L.bind_attention(x, _rows(8, 128, norm=True))
    L.bind_attention(x, _rows(8, 128))


def test_layers_with_plain_experts_refuse_8bit_weights(layer):
    """A plain layer's, an 8-bit cache's and a stack's block alike."""
    from paper_2606_15615_amd import _lib
    from paper_2606_15615_amd.layer import MoecaLayer
    p = _lib.moeca_policy_default()
    p.batch, p.tokens = 1, 8
    stack = _lib.moeca_stack_create(2, 128, 2, 4, 2, 64, p)
    try:
        block = MoecaLayer.attach(_lib.moeca_stack_layer(stack, 1), _bytes(16), 128, 4, 2, 64,
                                  batch=1, tokens=8)
        for L in (layer(n_shared=0), layer(cache="e4m3"), block):
            with pytest.raises(_lib.MoecaError, match="not quantised"):
                L.set_weights_quant(_bytes(4, 256), None, _stack(4, 64, 128), _stack(4, 128, 64))
    finally:
        _lib.moeca_stack_destroy(stack)
