"""The 8-bit entry points on the host: sizes, refusals and what a change of a
layer's quantisation undoes, without launching GPU work."""
import pytest

FAKE = 1 << 40  # never dereferenced: the calls below fail, or do nothing, on the host
OK, INVAL, STATE = 0, -1, -2


@pytest.fixture(scope="module")
def L():
    from paper_2606_15615_amd import _lib
    _lib.load()
    return _lib


def _pol(L, **kw):
    p = L.moeca_policy_default()
    p.batch, p.tokens = 2, 16
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("K,pitch,scales", [
    (1, 128, 16), (128, 128, 16), (129, 256, 16), (1152, 1152, 16), (2048, 2048, 16),
    (2049, 2176, 32), (1 << 20, 1 << 20, 8192), (0, 0, 0), (-5, 0, 0)])
def test_pitches(L, K, pitch, scales):
    assert L.moeca_quant_pitch(K) == pitch
    assert L.moeca_quant_scale_pitch(K) == scales
    if K > 0:
        assert L.moeca_quant_linear_bytes(3, K) >= 3 * (pitch + scales)
    assert L.moeca_quant_linear_bytes(0, K) == 0


ROWS = dict(src=FAKE, dtype=0, rows=4, K=200, ld=200, slot=FAKE, slots=9, q=FAKE, scale=FAKE,
            norm=FAKE)


@pytest.mark.parametrize("kw", [
    dict(src=None), dict(dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(K=0),
    dict(K=(1 << 20) + 1, ld=1 << 21), dict(ld=199), dict(slots=-1), dict(slots=1 << 31),
    dict(slot=None, slots=3), dict(q=None), dict(scale=None), dict(q=FAKE + 8),
    dict(scale=FAKE + 4), dict(slot=FAKE + 2), dict(norm=FAKE + 1), dict(src=FAKE + 1),
    dict(dtype=1, src=FAKE + 2)])
def test_quant_rows_refuses(L, kw):
    a = {**ROWS, **kw}
    assert L.load().moeca_quant_rows(*a.values(), None) == INVAL
    assert L.moeca_last_error() != ""


@pytest.mark.parametrize("kw", [
    dict(dst=None), dict(dtype=7), dict(rows=-2), dict(K=-1), dict(ld=100), dict(slots=-1),
    dict(slot=None, slots=3), dict(q=None), dict(scale=FAKE + 8), dict(slot=FAKE + 1),
    dict(dst=FAKE + 1)])
def test_dequant_rows_refuses(L, kw):
    a = dict(q=FAKE, scale=FAKE, slots=9, K=200, slot=FAKE, rows=4, dst=FAKE, dtype=0, ld=200)
    a.update(kw)
    assert L.load().moeca_dequant_rows(*a.values(), None) == INVAL
    assert L.moeca_last_error() != ""


@pytest.mark.parametrize("kw", [
    dict(W=None), dict(dtype=5), dict(count=-1), dict(count=65536), dict(N=0),
    dict(N=(1 << 20) + 1), dict(K=0), dict(q=None), dict(scale=None), dict(q=FAKE + 1),
    dict(W=FAKE + 1)])
def test_quant_matrix_refuses(L, kw):
    a = dict(W=FAKE, dtype=0, count=2, N=30, K=70, q=FAKE, scale=FAKE)
    a.update(kw)
    assert L.load().moeca_quant_matrix(*a.values(), None) == INVAL
    assert L.moeca_last_error() != ""


LINEAR = dict(x=FAKE, dtype=0, M=5, K=200, ldx=200, q=FAKE, scale=FAKE, N=70, bias=FAKE, out=FAKE,
              ldo=70, ws=FAKE, bytes=1 << 20)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(dtype=3), dict(M=-1), dict(K=0), dict(ldx=10), dict(q=None),
    dict(scale=None), dict(q=FAKE + 4), dict(N=0), dict(N=1 << 21, ldo=1 << 21), dict(out=None),
    dict(ldo=69), dict(out=FAKE + 1), dict(bias=FAKE + 2), dict(ws=None), dict(ws=FAKE + 16),
    dict(bytes=10), dict(M=1 << 30, N=1 << 20, ldo=1 << 20)])
def test_quant_linear_refuses(L, kw):
    a = {**LINEAR, **kw}
    assert L.load().moeca_quant_linear(*a.values(), None) == INVAL
    assert L.moeca_last_error() != ""


def test_nothing_to_do_is_no_error(L):
    lib = L.load()
    a = {**ROWS, "rows": 0, "src": None}
    assert lib.moeca_quant_rows(*a.values(), None) == OK
    a = {**ROWS, "slots": 0}
    assert lib.moeca_quant_rows(*a.values(), None) == OK
    assert lib.moeca_dequant_rows(None, None, 0, 5, None, 0, None, 0, 5, None) == OK
    assert lib.moeca_quant_matrix(None, 0, 0, 3, 5, None, None, None) == OK
    a = {**LINEAR, "M": 0, "x": None, "out": None, "ws": None, "bytes": 0}
    assert lib.moeca_quant_linear(*a.values(), None) == OK


def test_layer_quant_host_paths(L):
    lib = L.load()
    E, C = L.MOECA_QUANT_EXPERTS, L.MOECA_QUANT_CACHE
    h = L.moeca_layer_create(192, 8, 2, 320, _pol(L, n_shared=1))
    full = L.moeca_layer_create(192, 8, 2, 320, _pol(L, mode=L.MOECA_MODE_FULL))
    try:
        assert lib.moeca_layer_set_quant(None, 0) == INVAL
        assert lib.moeca_layer_set_quant(h, 4) == INVAL
        assert lib.moeca_layer_set_quant(full, C) == INVAL
        assert "no cache" in L.moeca_last_error()
        assert lib.moeca_layer_set_quant(full, E) == OK
        # calls of the other form are refused
        assert lib.moeca_layer_set_weights_quant(h, *[FAKE] * 6) == INVAL
        assert lib.moeca_layer_set_shared_quant(h, *[FAKE] * 4) == INVAL
        assert lib.moeca_bind_attention_quant(h, *[FAKE] * 3) == INVAL
        assert lib.moeca_layer_set_weights_quant(None, *[FAKE] * 6) == INVAL
        assert lib.moeca_layer_set_shared_quant(None, *[FAKE] * 4) == INVAL
        assert lib.moeca_bind_attention_quant(None, *[FAKE] * 3) == INVAL
        plain = L.moeca_workspace_bytes(h)
        assert L.moeca_layer_set_weights(h, FAKE, None, FAKE, FAKE) == OK
        assert L.moeca_layer_set_shared(h, FAKE, FAKE) == OK
        assert L.moeca_bind_workspace(h, FAKE, plain) == OK
        # nothing changes: what is bound stays
        assert lib.moeca_layer_set_quant(h, 0) == OK
        assert lib.moeca_step(h, None, 0, FAKE, None) == INVAL
        # the cache alone: the weights stay, workspace and attention go
        assert L.moeca_bind_attention(h, FAKE, FAKE) == OK
        assert lib.moeca_layer_set_quant(h, C) == OK
        assert lib.moeca_step(h, FAKE, 0, FAKE, None) == STATE
        assert "workspace" in L.moeca_last_error()
        assert lib.moeca_bind_attention(h, FAKE, FAKE) == INVAL
        assert lib.moeca_bind_attention(h, None, None) == OK
        assert lib.moeca_bind_attention_quant(h, FAKE, FAKE, None) == INVAL
        assert lib.moeca_bind_attention_quant(h, FAKE, FAKE, FAKE + 8) == INVAL
        assert lib.moeca_bind_attention_quant(h, FAKE, FAKE, FAKE) == OK
        n = 2 * 16 * 2
        assert L.moeca_debug_buffer(h, L.BUF["h_c"])[1] == n * 256
        assert L.moeca_debug_buffer(h, L.BUF["s_c"])[1] == n * 16
        # and the experts: the weights go
        assert lib.moeca_layer_set_quant(h, C | E) == OK
        nbytes = L.moeca_workspace_bytes(h)
        assert L.moeca_bind_workspace(h, FAKE, nbytes) == OK
        assert lib.moeca_step(h, FAKE, 0, FAKE, None) == STATE
        assert "weights" in L.moeca_last_error()
        assert lib.moeca_layer_set_weights(h, FAKE, None, FAKE, FAKE) == INVAL
        assert lib.moeca_layer_set_shared(h, FAKE, FAKE) == INVAL
        for bad in ([None] + [FAKE] * 5, [FAKE, None, None, FAKE, FAKE, FAKE],
                    [FAKE + 8, None] + [FAKE] * 4, [FAKE, FAKE + 2] + [FAKE] * 4,
                    [FAKE, None, FAKE, FAKE + 4, FAKE, FAKE]):
            assert lib.moeca_layer_set_weights_quant(h, *bad) == INVAL
        assert lib.moeca_layer_set_weights_quant(h, FAKE, None, *[FAKE] * 4) == OK
        assert lib.moeca_step(h, FAKE, 0, FAKE, None) == STATE
        assert "shared" in L.moeca_last_error()
        assert lib.moeca_forward_noalloc(h, FAKE, 1, FAKE, None) == STATE
        assert lib.moeca_layer_set_shared_quant(h, FAKE, FAKE, FAKE, None) == INVAL
        assert lib.moeca_layer_set_shared_quant(h, FAKE + 8, FAKE, FAKE, FAKE) == INVAL
        assert lib.moeca_layer_set_shared_quant(full, *[FAKE] * 4) == INVAL
        assert lib.moeca_layer_set_shared_quant(h, *[FAKE] * 4) == OK
        assert lib.moeca_step(h, None, 0, FAKE, None) == INVAL
        # buffers: inside the workspace, aligned, disjoint
        spans = sorted(L.moeca_debug_buffer(h, i) for i in range(len(L.BUF)))
        for (o1, b1), (o2, _) in zip(spans, spans[1:]):
            assert o1 % 256 == 0 and o1 + b1 <= o2
        assert spans[-1][0] + spans[-1][1] <= nbytes
        # back to the plain form: the sizes of before
        assert lib.moeca_layer_set_quant(h, 0) == OK
        assert L.moeca_workspace_bytes(h) == plain
        assert lib.moeca_step(h, FAKE, 0, FAKE, None) == STATE
    finally:
        L.moeca_layer_destroy(h)
        L.moeca_layer_destroy(full)


def test_a_stacks_layer_is_refused(L):
    lib = L.load()
    s = L.moeca_stack_create(2, 576, 8, 4, 2, 256, _pol(L))
    try:
        layer = L.moeca_stack_layer(s, 1)
        assert lib.moeca_layer_set_quant(layer, L.MOECA_QUANT_EXPERTS) == STATE
        assert "stack" in L.moeca_last_error()
    finally:
        L.moeca_stack_destroy(s)


def test_python_refusals():
    """What the binding refuses before any call: shapes, types, strides, devices."""
    import torch
    from paper_2606_15615_amd import quant
    r = quant.QuantRows(6, 200, device="cpu", norm=True)
    assert r.q.shape == (6, 256) and r.scale.shape == (6, 16) and r.norm.shape == (6,)
    with pytest.raises(ValueError, match="width 200"):
        r.write(torch.zeros(3, 199))
    with pytest.raises(ValueError, match="contiguous"):
        r.write(torch.zeros(200, 3).T)
    with pytest.raises(ValueError, match="overlap"):
        r.write(torch.zeros(200).expand(3, 200))
    with pytest.raises(ValueError, match="expected cpu"):
        r.write(torch.zeros(3, 200, device="meta"))
    with pytest.raises(ValueError, match="2 slots for 3 rows"):
        r.write(torch.zeros(3, 200), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="int32"):
        r.write(torch.zeros(3, 200), torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="out has"):
        r.read(out=torch.zeros(5, 200))
    with pytest.raises(TypeError):
        r.read(dtype=torch.bfloat16, out=torch.zeros(6, 200))
    assert r.read(torch.zeros(0, dtype=torch.int32)).shape == (0, 200)
    r.write(torch.zeros(0, 200))
    with pytest.raises(ValueError, match="come together"):
        quant.QuantRows(2, 5, q=torch.zeros(2, 128, dtype=torch.uint8))
    with pytest.raises(ValueError, match="scale"):
        quant.QuantRows(2, 5, q=torch.zeros(2, 128, dtype=torch.uint8),
                        scale=torch.zeros(2, 1, dtype=torch.uint8))
    with pytest.raises(ValueError, match="norm"):
        quant.QuantRows(2, 5, device="cpu", norm=torch.zeros(3))
    q, s = torch.zeros(70, 256, dtype=torch.uint8), torch.zeros(1, 16, dtype=torch.uint8)
    W = quant.QuantMatrix(q, s, 70, 200)
    with pytest.raises(ValueError, match="q:"):
        quant.QuantMatrix(q, s, 71, 200)
    with pytest.raises(ValueError, match="scale:"):
        quant.QuantMatrix(q, torch.zeros(2, 16, dtype=torch.uint8), 70, 200)
    with pytest.raises(ValueError, match="stack"):
        quant.linear(torch.zeros(1, 200), quant.QuantMatrix(q[None], s[None], 70, 200))
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        quant.linear(torch.zeros(1, 200, dtype=torch.float16), W)
    with pytest.raises(TypeError, match="out is"):
        quant.linear(torch.zeros(1, 200), W, out=torch.zeros(1, 70, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="bias"):
        quant.linear(torch.zeros(1, 200), W, bias=torch.zeros(69))
    with pytest.raises(ValueError, match="rows, x"):
        quant.linear(torch.zeros(1, 200), W, out=torch.zeros(2, 70))
    assert quant.linear(torch.zeros(0, 200), W).shape == (0, 70)
    with pytest.raises(ValueError, match="contiguous"):
        quant.quantize_matrix(torch.zeros(8, 4).T)


def test_host_tensors_are_refused():
    import torch
    from paper_2606_15615_amd import quant
    r = quant.QuantRows(3, 20, device="cpu")
    with pytest.raises(ValueError, match="not on a GPU"):
        r.write(torch.zeros(2, 20))
    with pytest.raises(ValueError, match="not on a GPU"):
        r.read()
    with pytest.raises(ValueError, match="not on a GPU"):
        quant.quantize_matrix(torch.zeros(2, 20))
    W = quant.QuantMatrix(torch.zeros(70, 256, dtype=torch.uint8),
                          torch.zeros(1, 16, dtype=torch.uint8), 70, 200)
    with pytest.raises(ValueError, match="not on a GPU"):
        quant.linear(torch.zeros(1, 200), W)
