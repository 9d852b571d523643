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


def test_results_on_another_stream():
    """Results that a call on a side stream makes are not memory that the busy current
    stream still uses: blocks it has just given back keep their last readers."""
    import torch
    from paper_2606_15615_amd import quant
    g = torch.Generator(device="cuda:0")
    g.manual_seed(4)
    x = torch.randn(500, 640, generator=g, device="cuda:0").bfloat16()
    W = quant.quantize_matrix(torch.randn(384, 640, generator=g, device="cuda:0"))
    ws = quant.linear_workspace(500, 640)
    rows = quant.QuantRows(500, 640)
    rows.write(x)
    big = torch.randn(2048, 2048, generator=g, device="cuda:0") / 45
    want = quant.linear(x, W), rows.read()
    side = torch.cuda.Stream()
    for call, ref in ((lambda: quant.linear(x, W, workspace=ws, stream=side), want[0]),
                      (lambda: rows.read(stream=side), want[1])):
        for _ in range(3):
            torch.cuda.synchronize()
            _busy(big)
            old = torch.full_like(ref, 3.0)      # late, on the current stream
            seen = old + 1
            del old
            got = call()
            torch.cuda.synchronize()
            assert torch.equal(got, ref) and bool((seen == 4.0).all())
            del got, seen


def _layer(d, E, k, d_ff, B, N, seed=0, dtype="bf16", bias=False, **kw):
    """A layer with random weights, 8-bit where it is asked for, and its input."""
    import torch
    from paper_2606_15615_amd import quant
    from paper_2606_15615_amd.layer import MoecaLayer
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)

    def rnd(*s):
        t = torch.randn(*s, generator=g, device="cuda:0")
        return t.bfloat16() if dtype == "bf16" else t
    L = MoecaLayer(d, E, k, d_ff, batch=B, tokens=N, dtype=dtype, **kw)
    U = L.up_rows
    w = [rnd(E, U, d) / d ** 0.5, rnd(E, d, d_ff) / d_ff ** 0.5]
    put = L.set_weights
    if L.experts8:
        w, put = [quant.quantize_matrix(m) for m in w], L.set_weights_quant
    put(rnd(E, d) / d ** 0.5, None, *w)
    if L.n_shared:
        s = [rnd(L.n_shared, U, d) / d ** 0.5, rnd(L.n_shared, d, d_ff) / d_ff ** 0.5]
        (L.set_shared_quant(*map(quant.quantize_matrix, s)) if L.experts8 else L.set_shared(*s))
    L.reset()
    return L, rnd(B, N, d)


def test_a_device_without_an_index():
    """"cuda" is the current device: the same results as on "cuda:0"."""
    import torch
    from paper_2606_15615_amd import quant
    ys = []
    for device in ("cuda:0", "cuda"):
        L, x = _layer(192, 4, 2, 128, 1, 50, device=device, experts="e4m3", cache="e4m3")
        att = quant.QuantRows(50, 192, device=device)
        L.bind_attention(x, att)
        y = torch.zeros_like(x)
        L.step(x, 0, y)
        ys.append((y, att.q))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*ys))


@pytest.mark.parametrize("kw", [
    dict(d=256, E=8, k=2, d_ff=448, B=2, N=120),
    dict(d=192, E=4, k=3, d_ff=320, B=1, N=90, act="swiglu", n_shared=1),
    dict(d=640, E=4, k=2, d_ff=1088, B=1, N=900)])
@pytest.mark.parametrize("cache", [None, "e4m3"])
def test_noalloc_is_the_full_step(kw, cache):
    """moeca_forward_noalloc computes what a full step does, with the products that the
    layer's hidden rows take (exact ones where its cache is in 8 bits)."""
    import torch
    from paper_2606_15615_amd import _lib
    say(f"  {kw} cache {cache}")
    L, x = _layer(**kw, seed=5, experts="e4m3", cache=cache)
    y, z = torch.zeros_like(x), torch.zeros_like(x)
    L.step(x, 0, y)
    _lib.moeca_forward_noalloc(L.h, x.data_ptr(), L.B, z.data_ptr(),
                               torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert L.stats().full_step == 1
    assert torch.equal(y, z)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,N", [(256, 1), (256, 60), (384, 700), (640, 4000)])
def test_rows_of_an_8bit_cache_have_exact_products(n, N, dtype):
    """Every eight consecutive products hold 448 * 448 and its negative besides small
    integers, which instructions that align them to the largest and keep 2^-13 of it
    would lose.  All sums are integers below 2^24, so fp32 has them exactly in any
    order; large hidden values are their own GELU.  Output and cache are then known
    to the bit: the integers, rounded once to the type."""
    import torch
    from paper_2606_15615_amd import _lib, quant
    from paper_2606_15615_amd.layer import MoecaLayer
    say(f"  {N} tokens of {n} {dtype}")
    g = np.random.default_rng(n + N)
    x = g.integers(8, 16, (N, n)) * 2.0                   # 16 .. 30: e4m3 numbers
    x[:, ::8] = x[:, 4::8] = 448.0
    down = g.integers(-2, 3, (2, n, n)).astype(float)
    down[:, :, ::8], down[:, :, 4::8] = 448.0, -448.0
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    L = MoecaLayer(n, 2, 1, n, batch=1, tokens=N, dtype=dtype, experts="e4m3", cache="e4m3")
    eye = torch.eye(n, device="cuda:0", dtype=t).expand(2, n, n).contiguous()
    W_r = torch.from_numpy(g.normal(size=(2, n))).cuda().to(t)
    L.set_weights_quant(W_r, None, quant.quantize_matrix(eye),
                        quant.quantize_matrix(torch.from_numpy(down).cuda().to(t)))
    L.reset()
    xt = torch.from_numpy(x).cuda().to(t)[None]
    y, z = torch.zeros_like(xt), torch.zeros_like(xt)
    L.step(xt, 0, y)
    _lib.moeca_forward_noalloc(L.h, xt.data_ptr(), 1, z.data_ptr(),
                               torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    e = L.read("e_t")
    h = np.einsum("nd,nkd->nk", x, down[e]) if N <= 60 else np.where(
        (e == 0)[:, None], x @ down[0].T, x @ down[1].T)
    assert np.abs(h).max() < 2 ** 15
    h = torch.from_numpy(h).to(t)
    assert torch.equal(y[0].cpu(), h) and torch.equal(z, y)
    got = L.cache_rows().read(dtype=torch.float32).double().cpu().numpy()
    np.testing.assert_array_equal(got, Q.round_trip(h.double().numpy()))


U32 = 2.0 ** -24


@pytest.mark.parametrize("M,dtype", [(6, "fp32"), (6, "bf16"), (16, "bf16"), (70, "fp32"),
                                     (700, "fp32")])
def test_exact_products_at_the_least_scale(M, dtype):
    """Rows with the scale 2^-124 and every e4m3 number down to its subnormals, 2^-133
    in all: the least elements of which products are exact.  All are wanted to within
    the fp32 sums, K + 8 of half an ulp each of the magnitudes' sum, and one rounding."""
    import torch
    from paper_2606_15615_amd import quant
    K, N = 640, 200
    g = np.random.default_rng(M)
    x = Q.TABLE[g.integers(0, 127, (M, K))]
    x = np.where(g.random((M, K)) < 0.5, Q.TABLE[g.integers(0, 8, (M, K))], x)  # subnormals
    x[:, ::128] = 448.0
    x[0] = np.where(np.arange(K) % 128 == 0, 448.0, 2.0 ** -9)
    x *= np.where(g.random((M, K)) < 0.5, -1.0, 1.0) * 2.0 ** -124
    w = g.normal(size=(N, K)) / 2
    w[:, ::128] = 0                     # the largest elements meet nothing
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    xt = torch.from_numpy(x).to(t).cuda()
    np.testing.assert_array_equal(xt.double().cpu().numpy(), x)
    wt = torch.from_numpy(w).cuda().to(torch.bfloat16)
    q, s = Q.quant_rows(x)
    assert (s == 3).all()
    wv = Q.matrix_values(*Q.quant_matrix(wt.double().cpu().numpy()), K)
    want, mag = x @ wv.T, np.abs(x) @ np.abs(wv).T
    got = quant.linear(xt, quant.quantize_matrix(wt)).double().cpu().numpy()
    half = 2.0 ** -8 if dtype == "bf16" else U32
    # and half a step of the types' subnormals (2^-149, 2^-133)
    least = 2.0 ** (-134 if dtype == "bf16" else -150)
    tol = (K + 8) * (U32 * mag + 2.0 ** -150) + half * np.abs(want) + least
    say(f"  {M} rows {dtype}: largest share of the bound {float((np.abs(got - want) / tol).max()):.3f}")
    assert np.all(np.abs(got - want) <= tol)


@pytest.mark.parametrize("k,d", [(2, 320), (2, 1152), (3, 192)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_buffers_at_odd_multiples_of_16_bytes(dtype, k, d):
    """The C calls want 16-byte alignment and no more: attention features, input,
    output and attention cache at 16 modulo 32."""
    import torch
    from paper_2606_15615_amd import quant
    say(f"  {dtype} k {k} d {d}")
    N = 45

    def shifted(n, t):
        size = torch.empty(0, dtype=t).element_size()
        b = torch.zeros(n * size + 48, dtype=torch.uint8, device="cuda:0")
        at = (16 - b.data_ptr()) % 32
        b = b[at:at + n * size].view(t)
        assert b.data_ptr() % 32 == 16
        return b
    L, x = _layer(d, 4, k, 128, 1, N, seed=d, dtype=dtype, experts="e4m3", cache="e4m3")
    g = torch.Generator(device="cuda:0")
    g.manual_seed(1)
    a = torch.randn(N, d, generator=g, device="cuda:0").to(x.dtype)
    got = []
    for off in (False, True):
        xs, ys, at = x, torch.zeros_like(x), a
        rows = quant.QuantRows(N, d)
        if off:
            xs, ys, at = (shifted(N * d, x.dtype).view(1, N, d) for _ in range(3))
            xs.copy_(x), at.copy_(a)
            rows = quant.QuantRows(N, d, q=shifted(N * rows.pitch, torch.uint8).view(N, -1),
                                   scale=shifted(N * rows.scale_pitch, torch.uint8).view(N, -1))
        L.bind_attention(at, rows)
        L.reset()
        L.step(xs, 0, ys)
        torch.cuda.synchronize()
        got.append((ys.clone(), rows.q.clone(), rows.scale[:, :-(-d // 128)].clone(),
                    rows.read()))
    assert all(torch.equal(u, v) for u, v in zip(*got))
    q, s = Q.quant_rows(a.double().cpu().numpy())
    np.testing.assert_array_equal(got[1][1].cpu().numpy(), q)
    np.testing.assert_array_equal(got[1][2].cpu().numpy(), s)
