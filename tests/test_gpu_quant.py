"""8-bit rows, matrices, products and layers on the GPU against the 64-bit oracle
(oracle/quant_oracle.py).

Quantising is exact: elements, scales and read-back values are compared bit for
bit.  A product has exact operands, so a result may be off by the fp32 sums and
one rounding: |y - y64| <= half an ulp of the type + (n + 8) 2^-24 sum |x w|
for n summed terms, and, where the 8-bit matrix instructions are used (bf16
results), 2^-13 of the largest product of each group of eight k, which is at most
2^-13 sum |x w|.  Hidden rows that are quantised inside a layer may lie anywhere
between the oracle's neighbours of their bound (quant_oracle.neighbours), and
what follows is bounded by the products' sum over that width.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import moeca_oracle as O
from oracle import quant_oracle as Q

U32, U16 = 2.0 ** -24, 2.0 ** -8   # half an ulp, relative
GROUP = 2.0 ** -13


def say(msg):
    print(msg, flush=True)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_15615_amd import _lib
    _lib.load()


def _t(a, dtype="fp32"):
    """A numpy array on the GPU in this type, and its exact values."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0", torch.float32)
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    return t, t.double().cpu().numpy()


def _rows(g, R, K):
    x = g.normal(size=(R, K)) * np.exp(g.normal(size=(R, 1)) * 2)
    return np.where(g.random((R, K)) < 0.01, x * 20, x)


def _strided(t, extra):
    """The same values in rows `extra` elements further apart."""
    import torch
    big = torch.full((t.shape[0], t.shape[1] + extra), 7.0, dtype=t.dtype, device=t.device)
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]], big


# ---- rows ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("R,K,extra", [(1, 1, 0), (3, 64, 0), (5, 127, 1), (4, 128, 8), (7, 129, 0),
                                       (300, 1000, 24), (2, 1152, 3), (33, 4608, 0), (1, 20000, 0)])
def test_write_and_read(R, K, extra, dtype):
    import torch
    from paper_2606_15615_amd import quant
    say(f"  write {R} x {K} stride +{extra} {dtype}")
    g = np.random.default_rng(R * 7919 + K)
    x, x64 = _t(_rows(g, R, K), dtype)
    if extra:
        x, _ = _strided(x, extra)
    slots = R + 3
    slot = g.permutation(slots)[:R].astype(np.int32)
    if R > 2:
        slot[1], slot[2] = -1, slots     # left out
    keep = (slot >= 0) & (slot < slots)
    c = quant.QuantRows(slots, K, norm=True)
    c.q.fill_(0x55), c.scale.fill_(99), c.norm.fill_(-3.0)
    st = torch.from_numpy(slot).cuda()
    c.write(x, st)
    q, s = Q.quant_rows(x64[keep])
    nb = s.shape[1]
    wq = np.full((slots, c.pitch), 0x55, np.uint8)
    ws = np.full((slots, nb), 99, np.uint8)
    wn = np.full(slots, -3.0)
    wq[slot[keep]], ws[slot[keep]] = q, s
    val = Q.row_values(q, s, K)
    wn[slot[keep]] = np.sqrt((val * val).sum(1))
    np.testing.assert_array_equal(c.q.cpu().numpy(), wq)
    np.testing.assert_array_equal(c.scale.cpu().numpy()[:, :nb], ws)
    # one rounding of an fp64 sum to fp32
    np.testing.assert_allclose(c.norm.cpu().numpy(), wn, rtol=1.01 * U32, atol=0)

    out = torch.full((R, K + extra), 9.0, dtype=x.dtype, device="cuda:0")
    c.read(st, out=out[:, :K])
    want = np.zeros((R, K))
    want[keep] = val
    got = out.double().cpu().numpy()
    np.testing.assert_array_equal(got[:, :K], want)   # four bits fit either type
    assert (got[:, K:] == 9.0).all()
    allr = c.read(dtype=torch.float32).double().cpu().numpy()
    np.testing.assert_array_equal(allr[slot[keep]], val)


def test_special_values():
    """Empty blocks, subnormals, the borders of a scale, the largest numbers, ties,
    NaN and infinities; -0 keeps its sign."""
    import torch
    from paper_2606_15615_amd import quant
    big = float(np.finfo(np.float32).max)
    rows = np.zeros((14, 256), np.float32)
    rows[1, :4] = [1e-45, -1e-45, 1.2e-38, -0.0]
    rows[2, :3] = [448.0, 1.0, 2.0 ** -10]
    rows[3, :3] = [np.nextafter(np.float32(448), np.float32(500)), 1.0, 2.0 ** -9 * 3]
    rows[4, 0] = big
    rows[5, 5] = -big
    rows[6, :5] = [np.nan, 3.0, -np.nan, 0.1, 5.0]
    rows[7, :5] = [np.inf, 3.0, -np.inf, 0.1, 5.0]
    rows[8] = np.inf
    rows[9, :128] = (np.arange(128) - 64) / 16.0 + 1 / 32        # ties among the mantissas
    rows[10, :128] = 448 * 2.0 ** -np.arange(128)
    rows[11, 128:] = 2.0 ** -126
    rows[12] = np.float32(2.0 ** 127)
    rows[13, ::2] = -0.0
    c = quant.QuantRows(14, 256, norm=True)
    c.write(torch.from_numpy(rows).cuda())
    q, s = Q.quant_rows(rows.astype(np.float64))
    gq = c.q.cpu().numpy()
    nan = (q & 0x7F) == 0x7F
    np.testing.assert_array_equal((gq & 0x7F) == 0x7F, nan)
    np.testing.assert_array_equal(gq[~nan], q[~nan])
    np.testing.assert_array_equal(c.scale.cpu().numpy()[:, :2], s)
    with np.errstate(over="ignore"):
        want = Q.row_values(q, s, 256).astype(np.float32)
    np.testing.assert_array_equal(c.read(dtype=torch.float32).cpu().numpy(), want)
    n = c.norm.cpu().numpy()
    assert np.isnan(n[6]) and np.isnan(n[7]) and np.isnan(n[8]) and n[0] == 0.0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,N,K", [(1, 1, 1), (1, 128, 128), (2, 129, 257), (3, 200, 1000),
                                   (1, 1152, 640)])
def test_matrix(n, N, K, dtype):
    from paper_2606_15615_amd import quant
    say(f"  matrix {n} x {N} x {K} {dtype}")
    g = np.random.default_rng(N + K)
    w, w64 = _t(g.normal(size=(n, N, K)) / np.sqrt(K), dtype)
    m = quant.quantize_matrix(w if n > 1 else w[0].contiguous())
    for i in range(n):
        q, s = Q.quant_matrix(w64[i])
        gq, gs = (m.q[i], m.scale[i]) if n > 1 else (m.q, m.scale)
        np.testing.assert_array_equal(gq.cpu().numpy(), q)
        np.testing.assert_array_equal(gs.cpu().numpy()[:, :s.shape[1]], s)


# ---- products -------------------------------------------------------------------
def _linear_bound(x, w, y, dtype, K):
    mag = np.abs(x) @ np.abs(w).T
    tol = (K + 8) * U32 * mag + (U16 if dtype == "bf16" else U32) * np.abs(y)
    return tol + (GROUP * mag if dtype == "bf16" else 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,K,N,extra,bias", [
    (1, 1, 1, 0, False), (1, 1152, 4608, 0, True), (2, 64, 3, 1, True), (3, 129, 130, 0, False),
    (7, 1000, 257, 5, True), (15, 128, 64, 0, True), (16, 2304, 576, 8, False),
    (17, 640, 1000, 0, True), (33, 4608, 1152, 0, True), (64, 1152, 1728, 0, False),
    (65, 320, 70, 2, True), (129, 1000, 1730, 0, True), (200, 2100, 300, 0, False),
    (513, 1152, 1152, 0, True), (1000, 192, 2305, 4, False), (2049, 1280, 640, 0, True),
    # 17, 33, 31 and 4 blocks of K: pieces of 16 scales that end in the last blocks
    (300, 2100, 700, 0, True), (777, 4224, 130, 0, False), (700, 3968, 520, 0, True),
    (900, 512, 1100, 8, True), (5000, 640, 2500, 0, True)])
def test_linear(M, K, N, extra, bias, dtype):
    import torch
    from paper_2606_15615_amd import quant
    say(f"  linear {M} x {K} x {N} stride +{extra} bias {bias} {dtype}")
    g = np.random.default_rng(M * 31 + K * 7 + N)
    x, x64 = _t(_rows(g, M, K), dtype)
    w, w64 = _t(g.normal(size=(N, K)) / np.sqrt(K), "bf16")
    b, b64 = _t(g.normal(size=N)) if bias else (None, 0.0)
    W = quant.quantize_matrix(w)
    wv = Q.matrix_values(*Q.quant_matrix(w64), K)
    xv = Q.round_trip(x64)
    out, big = None, None
    if extra:
        x, _ = _strided(x, extra)
        big = torch.full((M, N + extra), 9.0, dtype=x.dtype, device="cuda:0")
        out = big[:, :N]
    y = quant.linear(x, W, b, out=out)
    want = xv @ wv.T + b64
    got = y.double().cpu().numpy()
    err, tol = np.abs(got - want), _linear_bound(xv, wv, want, dtype, K) + U32 * np.abs(want)
    say(f"    largest share of the bound {float((err / np.maximum(tol, 1e-300)).max()):.3f}")
    assert np.all(err <= tol)
    if big is not None:
        assert bool((big[:, N:] == 9.0).all())
    # the same call gives the same bits, and a row alone the bound of its own
    assert torch.equal(quant.linear(x, W, b), y)
    one = quant.linear(x[M - 1:], W, b).double().cpu().numpy()
    assert np.all(np.abs(one - want[M - 1:]) <= tol[M - 1:])


def test_linear_special_rows():
    """NaN stays in its row; a zero row gives the bias; scales far apart do not meet."""
    import torch
    from paper_2606_15615_amd import quant
    g = np.random.default_rng(5)
    for M in (6, 200):
        x = g.normal(size=(M, 300)).astype(np.float32)
        x[1, 7] = np.nan
        x[2] = 0
        x[3] *= 2.0 ** 60
        x[4] *= 2.0 ** -60
        w, w64 = _t(g.normal(size=(140, 300)), "bf16")
        b, b64 = _t(g.normal(size=140))
        for dt in (torch.float32, torch.bfloat16):
            xt = torch.from_numpy(x).cuda().to(dt)
            y = quant.linear(xt, quant.quantize_matrix(w), b).double().cpu().numpy()
            assert np.isnan(y[1]).all() and not np.isnan(np.delete(y, 1, 0)).any()
            xv = Q.round_trip(np.delete(xt.double().cpu().numpy(), 1, 0))
            wv = Q.matrix_values(*Q.quant_matrix(w64), 300)
            want = xv @ wv.T + b64
            tol = _linear_bound(xv, wv, want, "bf16" if dt == torch.bfloat16 else "fp32", 300)
            assert np.all(np.abs(np.delete(y, 1, 0) - want) <= tol + U32 * np.abs(want))
            assert np.all(np.abs(y[2] - b64) <= U16 * np.abs(b64) if dt == torch.bfloat16
                          else y[2] == b64)


# ---- layers ---------------------------------------------------------------------
def _act64(z, act):
    if act == "swiglu":
        return O.silu(z[:, 0::2]) * z[:, 1::2]
    return O.gelu(z, act)


def _hidden(x, wup, act, exact):
    """Hidden values and how far the fp32 ones may be from them."""
    z = x @ wup.T
    dz = ((x.shape[1] + 8) * U32 + (0 if exact else GROUP)) * (np.abs(x) @ np.abs(wup).T)
    m = _act64(z, act)
    # |act'| <= 1.13; the exponential's argument carries |u| ulps, u <= 1.6 |z| (1 + z^2 / 22);
    # six more roundings
    if act == "swiglu":
        gt, up, dg, du = z[:, 0::2], z[:, 1::2], dz[:, 0::2], dz[:, 1::2]
        return m, 1.13 * dg * (np.abs(up) + du) + (np.abs(O.silu(gt)) + 1.13 * dg) * du + \
            np.abs(m) * (np.abs(gt) + 6) * 4 * U32
    u = np.abs(z) * (1 + z * z / 22)
    return m, 1.13 * dz + np.abs(m) * (2 * u + 8) * 4 * U32 + 2 * U32 * np.abs(z)


def _ffn(x, wup, wdown, act, exact, dtype):
    """An 8-bit expert's rows in 64 bits and the bound of the GPU's."""
    m, dm = _hidden(x, wup, act, exact)
    mid = Q.round_trip(m)
    lo, hi = Q.neighbours(m - dm, m + dm)
    wide = np.maximum(hi - mid, mid - lo)
    h = mid @ wdown.T
    mag = (np.abs(mid) + wide) @ np.abs(wdown).T
    tol = wide @ np.abs(wdown).T + ((m.shape[1] + 8) * U32 +
                                    (GROUP if dtype == "bf16" else 0)) * mag
    half = U16 if dtype == "bf16" else U32
    return h, tol + half * (np.abs(h) + tol)


class Case:
    """An 8-bit layer on the GPU with the oracle's view of its weights."""

    def __init__(self, d, E, k, d_ff, B, N, act="gelu_tanh", dtype="bf16", S=0, mode="ratio",
                 experts=True, cache=True, seed=0, attention=True, **pol):
        import torch
        from paper_2606_15615_amd import _lib, quant
        from paper_2606_15615_amd.layer import MoecaLayer
        modes = {"full": _lib.MOECA_MODE_FULL, "threshold": _lib.MOECA_MODE_THRESHOLD,
                 "ratio": _lib.MOECA_MODE_RATIO}
        self.d, self.E, self.k, self.B, self.N, self.act, self.S = d, E, k, B, N, act, S
        self.dtype, self.experts, self.cache, self.T = dtype, experts, cache, B * N
        self.mode = mode
        g = self.g = np.random.default_rng(seed)
        U = d_ff * (2 if act == "swiglu" else 1)
        self.L = MoecaLayer(d, E, k, d_ff, batch=B, tokens=N, mode=modes[mode], act=act,
                            dtype=dtype, n_shared=S, experts="e4m3" if experts else None,
                            cache="e4m3" if cache else None, **pol)

        def mats(n, rows, cols):
            w, w64 = _t(g.normal(size=(n, rows, cols)) / np.sqrt(cols), dtype)
            if not experts:
                return w, w64
            return quant.quantize_matrix(w), np.stack(
                [Q.matrix_values(*Q.quant_matrix(m), cols) for m in w64])

        W_r, _ = _t(g.normal(size=(E, d)) / np.sqrt(d), dtype)
        up, self.up = mats(E, U, d)
        down, self.down = mats(E, d, d_ff)
        (self.L.set_weights_quant if experts else self.L.set_weights)(W_r, None, up, down)
        if S:
            ups, self.ups = mats(S, U, d)
            downs, self.downs = mats(S, d, d_ff)
            (self.L.set_shared_quant if experts else self.L.set_shared)(ups, downs)
        self.attn = None
        if attention and mode != "full":
            self.attn_in = torch.zeros(B, N, d, device="cuda:0", dtype=self._dt())
            self.attn = (quant.QuantRows(B * N, d) if cache else torch.zeros_like(self.attn_in))
            self.L.bind_attention(self.attn_in, self.attn)
        self.L.reset()
        self.x = g.normal(size=(self.T, d))

    def _dt(self):
        import torch
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    def drift(self, share=0.05):
        self.x = np.sqrt(1 - share) * self.x + np.sqrt(share) * self.g.normal(size=self.x.shape)

    def state(self):
        rows = self.L.cache_rows()
        return dict(q=rows.q.cpu().numpy().copy(), s=rows.scale.cpu().numpy().copy(),
                    e=self.L.read("e_c"), n=self.L.read("n_c"), w=self.L.read("w_c"))

    def ffn(self, x64, up, down, exact):
        if self.experts:
            return _ffn(Q.round_trip(x64), up, down, self.act, exact, self.dtype)
        m, dm = _hidden(x64, up, self.act, True)
        half = U16 if self.dtype == "bf16" else U32
        dm = dm + half * np.abs(m)
        h = m @ down.T
        tol = dm @ np.abs(down).T + (m.shape[1] + 8) * U32 * (np.abs(m) @ np.abs(down).T)
        return h, tol + half * (np.abs(h) + tol)

    def step(self, t, label=""):
        """One step, checked against the oracle on the decisions the GPU took."""
        import torch
        T, k, d, cached = self.T, self.k, self.d, self.cache
        x, x64 = _t(self.x.reshape(self.B, self.N, d), self.dtype)
        x64 = x64.reshape(T, d)
        before = self.state() if cached else None
        if not cached and self.mode != "full":
            plain = self.L.read("h_c").reshape(T, k, d)
            if self.dtype == "bf16":
                plain = (plain.astype(np.uint32) << 16).view(np.float32)
        if self.attn is not None:
            a, a64 = _t(self.g.normal(size=(self.B, self.N, d)), self.dtype)
            self.attn_in.copy_(a)
            old_att = self.attn.q.cpu().numpy().copy() if cached else None
        y = torch.full_like(x, 9.0)
        self.L.step(x, t, y)
        torch.cuda.synchronize()
        e, w = self.L.read("e_t").reshape(T, k), self.L.read("w_t").reshape(T, k).astype(float)
        mask = self.L.read("mask").reshape(T, k) != 0
        sig = self.L.read("sigma").reshape(T, k)
        exact = self.dtype == "fp32" or cached
        h, tol = np.zeros((T, k, d)), np.zeros((T, k, d))
        for i in range(self.E):
            r, p = np.nonzero((e == i) & mask)
            if len(r):
                h[r, p], tol[r, p] = self.ffn(x64[r], self.up[i], self.down[i], exact)
        if cached or self.mode != "full":
            old = Q.row_values(before["q"], before["s"], d).reshape(T, k, d) if cached else plain
            r, p = np.nonzero(~mask)
            h[r, p] = old[r, sig[r, p]]
        want = (w[:, :, None] * h).sum(1)
        ytol = (w[:, :, None] * tol).sum(1)
        mag = (w[:, :, None] * np.abs(h)).sum(1)
        for i in range(self.S):
            hs, ts = self.ffn(x64, self.ups[i], self.downs[i], exact)
            want, ytol, mag = want + hs, ytol + ts, mag + np.abs(hs)
        half = U16 if self.dtype == "bf16" else U32
        ytol = ytol + (k + self.S + 2) * 2 * U32 * (mag + ytol)
        ytol = ytol + half * (np.abs(want) + ytol)
        got = y.double().cpu().numpy().reshape(T, d)
        err = np.abs(got - want)
        rel = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-30)
        say(f"    {label} t={t}: {int(mask.sum())} of {mask.size} recomputed, rel {rel:.2e}, "
            f"largest share of the bound {float((err / np.maximum(ytol, 1e-300)).max()):.3f}")
        assert np.all(err <= ytol)
        if not cached:
            return got, mask
        after = self.state()
        # reused slots untouched; written ones hold what the bound allows
        wrote = np.zeros((T, k), bool)
        r, p = np.nonzero(mask)
        wrote[r, sig[r, p]] = True
        flat = wrote.reshape(-1)
        np.testing.assert_array_equal(after["q"][~flat], before["q"][~flat])
        np.testing.assert_array_equal(after["s"][~flat], before["s"][~flat])
        np.testing.assert_array_equal(after["n"][~flat], before["n"][~flat])
        slot = r * k + sig[r, p]
        np.testing.assert_array_equal(after["e"][slot], e[r, p])
        np.testing.assert_array_equal(after["w"][slot].astype(float), w[r, p])
        val = Q.row_values(after["q"][slot], after["s"][slot], d)
        lo, hi = Q.neighbours(h[r, p] - tol[r, p], h[r, p] + tol[r, p])
        assert np.all((val >= lo) & (val <= hi))
        assert not after["q"][slot][:, d:].any()
        np.testing.assert_allclose(after["n"][slot], np.sqrt((val * val).sum(1)),
                                   rtol=1.01 * U32, atol=0)
        if self.attn is not None:
            sync = mask.any(1)
            q, s = Q.quant_rows(a64.reshape(T, d))
            aq, asc = self.attn.q.cpu().numpy(), self.attn.scale.cpu().numpy()
            np.testing.assert_array_equal(aq[sync], q[sync])
            np.testing.assert_array_equal(asc[sync][:, :s.shape[1]], s[sync])
            np.testing.assert_array_equal(aq[~sync], old_att[~sync])
        return got, mask


LAYERS = [
    dict(d=64, E=1, k=1, d_ff=64, B=1, N=1),
    dict(d=192, E=8, k=2, d_ff=320, B=2, N=77),
    dict(d=128, E=4, k=4, d_ff=128, B=1, N=50, act="gelu_erf"),
    dict(d=576, E=6, k=2, d_ff=448, B=2, N=150, act="swiglu"),
    dict(d=320, E=16, k=3, d_ff=192, B=3, N=61, act="swiglu", S=2),
    dict(d=256, E=64, k=8, d_ff=128, B=1, N=200, S=1),
    dict(d=256, E=5, k=2, d_ff=384, B=2, N=40, dtype="fp32"),
    dict(d=192, E=7, k=3, d_ff=192, B=1, N=90, dtype="fp32", act="swiglu", S=1),
    dict(d=640, E=3, k=2, d_ff=1088, B=1, N=700),
    dict(d=1152, E=2, k=1, d_ff=640, B=1, N=1100, act="gelu_erf"),
]


@pytest.mark.parametrize("form", ["both", "experts", "cache"])
@pytest.mark.parametrize("i", range(len(LAYERS)))
def test_layer(i, form):
    kw = LAYERS[i]
    say(f"  {form}: {kw}")
    c = Case(**kw, mode="ratio", ratio=0.4, experts=form != "cache", cache=form != "experts",
             seed=i)
    if form == "experts":
        c.attn = None
    for t in range(3):
        if form == "experts":
            # a plain cache: the layer's first (full) step only, others have their own tests
            if t == 0:
                c.step(t, form)
            continue
        _, mask = c.step(t, form)
        assert mask.all() == (t == 0) or c.T * c.k < 8
        c.drift()


@pytest.mark.parametrize("tau0,share", [(8.0, 0.01), (0.02, 0.3), (0.8, 0.1)])
def test_threshold_cycle(tau0, share):
    """Thresholds that recompute next to nothing, everything, and the default."""
    c = Case(384, 8, 2, 512, 2, 120, mode="threshold", tau0=tau0, seed=3)
    for t in range(5):
        c.step(t, f"tau0 {tau0}")
        c.drift(share)


@pytest.mark.parametrize("i", [0, 3, 4, 7, 8])
def test_uncached_and_noalloc(i):
    import torch
    from paper_2606_15615_amd import _lib
    kw = LAYERS[i]
    say(f"  uncached {kw}")
    c = Case(**kw, mode="full", cache=False, seed=20 + i)
    c.step(0, "full")
    x, _ = _t(c.x.reshape(c.B, c.N, c.d), c.dtype)
    y, z = torch.zeros_like(x), torch.zeros_like(x)
    c.L.step(x, 1, y)
    _lib.moeca_forward_noalloc(c.L.h, x.data_ptr(), c.B, z.data_ptr(),
                               torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(y, z)


def test_full_step_of_an_8bit_cache_is_the_plain_one():
    """A full step takes every row as the down projection left it: with plain
    experts its output is that of a layer with a plain cache, bit for bit."""
    import torch
    from paper_2606_15615_amd.layer import MoecaLayer
    g = torch.Generator(device="cuda:0")
    g.manual_seed(4)
    for E, k, d, d_ff, B, N in ((16, 2, 576, 2304, 2, 128), (8, 3, 320, 512, 1, 300)):
        def rnd(*s):
            return (torch.randn(*s, generator=g, device="cuda:0") / s[-1] ** 0.5).bfloat16()
        W = rnd(E, d), None, rnd(E, d_ff, d), rnd(E, d, d_ff)
        x = rnd(B, N, d) * d ** 0.5
        ys = []
        for cache in (None, "e4m3"):
            L = MoecaLayer(d, E, k, d_ff, batch=B, tokens=N, cache=cache)
            L.set_weights(*W)
            L.reset()
            y = torch.empty_like(x)
            L.step(x, 0, y)
            ys.append(y)
        torch.cuda.synchronize()
        # the K pieces of a plain cache are added by its combine, with the same order
        assert torch.equal(ys[0], ys[1])


def test_stream_and_graph():
    """A cycle on another stream, and replayed from a HIP graph with eager work
    between the replays: the bits of the eager run; two layers whose graphs run one
    after another keep apart."""
    import torch
    cases = [Case(256, 8, 2, 320, 2, 96, seed=s) for s in (1, 2)]
    xs, ys, want = [], [], []
    for c in cases:
        x = [_t(c.x.reshape(c.B, c.N, c.d), c.dtype)[0]]
        for _ in range(3):
            c.drift()
            x.append(_t(c.x.reshape(c.B, c.N, c.d), c.dtype)[0])
        xs.append(x)
        ys.append([torch.zeros_like(v) for v in x])

    def cycle(n):
        cases[n].L.reset()
        for t, (x, y) in enumerate(zip(xs[n], ys[n])):
            cases[n].L.step(x, t, y)

    for n in range(2):
        cycle(n)
        torch.cuda.synchronize()
        want.append([y.clone() for y in ys[n]] + [cases[n].L.cache_rows().q.clone()])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for n in range(2):
            for y in ys[n]:
                y.zero_()
            cycle(n)
    side.synchronize()
    for n in range(2):
        assert all(torch.equal(a, b) for a, b in zip(ys[n], want[n]))
    graphs = []
    for n in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            cycle(n)
        graphs.append(gr)
    for rep in range(4):
        for n in (0, 1) if rep % 2 else (1, 0):
            for y in ys[n]:
                y.fill_(5.0)
            graphs[n].replay()
        torch.cuda.synchronize()
        for n in range(2):
            got = ys[n] + [cases[n].L.cache_rows().q]
            assert all(torch.equal(a, b) for a, b in zip(got, want[n])), (rep, n)
        cases[rep % 2].L.stats()  # the program's own work between the replays


def test_rows_and_product_as_used_together():
    """Attention features go through the layer's 8-bit cache, are read back and
    projected, on one stream and in a graph."""
    import torch
    from paper_2606_15615_amd import quant
    c = Case(320, 4, 2, 256, 1, 130, seed=9)
    w, w64 = _t(c.g.normal(size=(200, 320)) / 18.0, "bf16")
    W = quant.quantize_matrix(w)
    ws = quant.linear_workspace(c.T, 320)
    feat = torch.empty(c.T, 320, dtype=torch.bfloat16, device="cuda:0")
    out = torch.empty(c.T, 200, dtype=torch.bfloat16, device="cuda:0")
    y = torch.empty(1, c.N, 320, dtype=torch.bfloat16, device="cuda:0")
    x, _ = _t(c.x.reshape(1, c.N, 320), "bf16")
    a, a64 = _t(c.g.normal(size=(c.T, 320)), "bf16")
    c.attn_in.copy_(a.view_as(c.attn_in))

    def run():
        c.L.reset()
        c.L.step(x, 0, y)
        c.attn.read(out=feat)
        quant.linear(feat, W, out=out, workspace=ws)

    run()
    torch.cuda.synchronize()
    f = Q.round_trip(a64)
    np.testing.assert_array_equal(feat.double().cpu().numpy(), f)
    # what was quantised once is quantised again without a change
    wv = Q.matrix_values(*Q.quant_matrix(w64), 320)
    want = f @ wv.T
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= _linear_bound(f, wv, want, "bf16", 320))
    keep = out.clone()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        run()
    for _ in range(3):
        out.zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, keep)


def test_far_slots():
    """Rows behind 4 GiB of elements: slot times pitch passes 32 bits."""
    import torch
    from paper_2606_15615_amd import quant
    slots, K = 1_100_000, 4096
    c = quant.QuantRows(slots, K)
    g = np.random.default_rng(8)
    x, x64 = _t(_rows(g, 3, K), "bf16")
    slot = torch.tensor([slots - 1, 0, 1_060_000], dtype=torch.int32, device="cuda:0")
    c.write(x, slot)
    np.testing.assert_array_equal(c.read(slot).double().cpu().numpy(), Q.round_trip(x64))
    assert int(c.q.view(torch.int32).count_nonzero()) <= 3 * K // 4


# ---- every tile -------------------------------------------------------------------
@pytest.mark.parametrize("M,K,N,extra,bias", [
    # five blocks of K, the fewest that the 256-column tiles are chosen for; 17, 31, 32
    # and 33: pieces of 16 scales; columns that end inside a half and unaligned rows
    (4000, 640, 3900, 0, True), (2049, 2176, 4609, 0, False), (3300, 3968, 2570, 6, True),
    (5000, 4096, 2307, 5, False), (3500, 4224, 2500, 12, True),
    # 128-row tiles
    (1000, 4608, 4608, 0, True), (8192, 700, 2050, 2, False)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_linear_many_rows(M, K, N, extra, bias, dtype):
    """The larger tiles; the 64-bit products are the GPU's own."""
    import torch
    from paper_2606_15615_amd import quant
    say(f"  linear {M} x {K} x {N} stride +{extra} bias {bias} {dtype}")
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(M + K + N)

    def rnd(*s):
        return torch.randn(*s, generator=gen, device="cuda:0")
    x = rnd(M, K) * torch.exp(2 * rnd(M, 1))
    x = x.bfloat16() if dtype == "bf16" else x
    w = (rnd(N, K) / K ** 0.5).bfloat16()
    b = rnd(N) if bias else None
    W = quant.quantize_matrix(w)
    rows = quant.QuantRows(M, K)
    rows.write(x)
    xv = rows.read(dtype=torch.float32).double()       # exact
    sc = W.scale[:, :(K + 127) // 128].double()
    wv = W.q.view(torch.float8_e4m3fn)[:, :K].double() * torch.exp2(
        sc.repeat_interleave(128, 1)[:, :K].repeat_interleave(128, 0)[:N] - 127)
    big = torch.full((M, N + extra), 9.0, dtype=x.dtype, device="cuda:0")
    out = big[:, :N]
    quant.linear(x, W, b, out=out)
    want = xv @ wv.t()
    mag = xv.abs() @ wv.abs().t()
    if bias:
        want += b.double()
    tol = (K + 9) * U32 * (mag + want.abs()) + (U16 if dtype == "bf16" else U32) * want.abs()
    if dtype == "bf16":
        tol += GROUP * mag
    err = (out.double() - want).abs()
    say(f"    largest share of the bound {float((err / tol).max()):.3f}")
    assert bool((err <= tol).all())
    assert bool((big[:, N:] == 9.0).all())


TILES = [
    # 256 x 256 tiles up and down, full ones and (threshold steps) 128 columns wide;
    # the 128-row tiles for exact products
    (dict(d=1536, E=8, k=2, d_ff=1536, B=1, N=4000), "experts"),
    (dict(d=1536, E=8, k=2, d_ff=1536, B=1, N=4000), "both"),
    (dict(d=640, E=8, k=2, d_ff=1472, B=1, N=4096, act="gelu_erf"), "experts"),
    # gated: 256 x 256, 128 x 256, and 128 x 256 exact; hidden widths that end in a block
    (dict(d=1664, E=8, k=2, d_ff=640, B=3, N=1100, act="swiglu", S=1), "experts"),
    (dict(d=1536, E=8, k=2, d_ff=768, B=1, N=4000, act="swiglu"), "both"),
    (dict(d=256, E=4, k=2, d_ff=192, B=1, N=400, act="swiglu"), "experts"),
    (dict(d=256, E=4, k=2, d_ff=320, B=1, N=400, act="swiglu", dtype="fp32"), "both"),
    # 128-row tiles, exact up and down
    (dict(d=640, E=8, k=2, d_ff=1280, B=2, N=1500, dtype="fp32"), "experts"),
    # small ones over a plain cache
    (dict(d=192, E=8, k=2, d_ff=320, B=2, N=77), "experts"),
    (dict(d=320, E=16, k=3, d_ff=192, B=3, N=61, act="swiglu", S=2), "experts"),
]


@pytest.mark.parametrize("i", range(len(TILES)))
def test_layer_tiles(i):
    """Full steps, steps that recompute next to nothing and steps that recompute
    most, over tiles of every size, with the plain and the 8-bit cache."""
    kw, form = TILES[i]
    say(f"  {form}: {kw}")
    c = Case(**kw, mode="threshold", tau0=8.0, cache=form == "both", seed=40 + i, attention=False)
    for t in range(3):
        c.step(t, form)
        c.drift(0.02 if t == 0 else 0.6)


def test_python_refusals_and_streams():
    """What the wrappers refuse before a launch; products on a stream of their own."""
    import torch
    from paper_2606_15615_amd import quant
    c = Case(128, 4, 2, 128, 1, 40, seed=1)
    plain = Case(128, 4, 2, 128, 1, 40, seed=1, cache=False)
    with pytest.raises(TypeError):
        c.L.bind_attention(c.attn_in, torch.zeros_like(c.attn_in))
    with pytest.raises(TypeError):
        plain.L.bind_attention(c.attn_in, c.attn)
    with pytest.raises(ValueError):
        c.L.bind_attention(c.attn_in, quant.QuantRows(39, 128))
    for args in ((c.attn_in, None), (None, c.attn)):
        with pytest.raises(Exception, match="NULL"):
            c.L.bind_attention(*args)
    with pytest.raises(ValueError):
        plain.L.cache_rows()
    c.L.bind_attention(None, None)
    c.attn = None
    c.step(0, "unbound")
    g = torch.Generator(device="cuda:0")
    g.manual_seed(2)
    W = quant.quantize_matrix(torch.randn(300, 500, generator=g, device="cuda:0"))
    side = torch.cuda.Stream()
    for M in (5, 70):
        xs = [torch.randn(M, 500, generator=g, device="cuda:0").bfloat16() for _ in range(2)]
        want = [quant.linear(x, W) for x in xs]
        with pytest.raises(ValueError):
            quant.linear(xs[0], W, stream=side)
        # two at a time, a workspace each
        ws = [quant.linear_workspace(M, 500) for _ in range(2)]
        out = [torch.zeros_like(w) for w in want]
        torch.cuda.synchronize()
        for _ in range(20):
            quant.linear(xs[0], W, out=out[0], workspace=ws[0])
            quant.linear(xs[1], W, out=out[1], workspace=ws[1], stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("d", [1984, 2112])
def test_wide_rows(d):
    """Rows of four groups of 512 elements, and of more."""
    c = Case(d, 4, 2, 64, 1, 60, mode="threshold", tau0=0.8, seed=d)
    for t in range(3):
        c.step(t, f"d {d}")
        c.drift(0.2)


def test_routing_to_one_expert():
    """Every token takes the same expert, the others have none."""
    import torch
    for act, B, N in (("gelu_tanh", 2, 900), ("swiglu", 1, 300)):
        c = Case(256, 8, 1, 192, B, N, act=act, mode="threshold", tau0=8.0, seed=6)
        c.x[:, :] = np.abs(c.x[:1]) + 0.01 * c.g.normal(size=c.x.shape)
        c.step(0, "one row of tokens")
        c.drift(0.001)
        c.step(1, "again")
