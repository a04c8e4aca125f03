"""Gated dense layers, dropout and the norms around a block against the float64 oracle.

Bars (relative L2 per output):
  float32   4e-6: a gated value is a product of two factors, each a sum and an activation like a dense
            layer's (2e-6 there); norms and sums over rows are those of the layer norm.
  bfloat16  against the float64 result rounded as the calls say (outputs once; a wide gated backward's dz
            before its products): what is left are single values whose float32 error crosses a tie, a step
            of 2^-8 to 2^-7 each: 3e-3, and one such step of a vector's largest among few values.
Masks are exact.
"""


import numpy as np
import pytest

from gpu_util import rel_l2
from oracle import blocks as ob, layers as ol
from test_gpu_layers import dev, e3, host, near_steps, out_like, packed, rounded  # noqa: F401 (e3: a fixture)

pytestmark = pytest.mark.gpu

DTS = ["float32", "bfloat16"]


def close(got, ref, dt, what="", bar=None):
    """got (on the device) is ref (float64) in type dt."""
    got, ref = host(got), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, what
    if ref.size == 0:
        return
    if dt == "float32":
        assert rel_l2(got, ref) < (bar or 4e-6), (what, rel_l2(got, ref))
        return
    ref = rounded(ref, dt)
    one = 2.0 ** -7 * np.abs(ref).max() / max(np.linalg.norm(ref), 1e-300)
    assert rel_l2(got, ref) < (bar or 3e-3) + (one if ref.size < 4000 else 0.0), (what, rel_l2(got, ref))


def names_of(e3, f):  # noqa: F811
    """The kernels that f launches."""
    import torch
    torch.cuda.synchronize()
    e3.timing_reset()
    e3.timing_enable(True)
    try:
        f()
        torch.cuda.synchronize()
        return set(e3.timing_read())
    finally:
        e3.timing_enable(False)
        e3.timing_reset()


# ---------------------------------------------------------------- gated dense layers
# M, K, N, gap, shift, and the kernel of the forward in float32 and in bfloat16
GATED = [(1, 1, 1, 0, 0, "few", "few"), (1, 4100, 40, 0, 0, "few", "few"), (7, 9001, 65, 1, 1, "few", "few"), (3, 2048, 2050, 0, 0, "few", "few"),
         (8, 2049, 3, 0, 0, "few", "few"), (8, 1500, 500, 4, 0, "few", "few"), (1, 1024, 100, 0, 0, "few", "few"), (2, 33, 31, 1, 1, "few", "few"),
         (3, 7, 64, 0, 0, "few", "few"), (8, 515, 129, 3, 0, "few", "few"), (5, 130, 8, 0, 3, "few", "few"),
         (9, 1, 1, 0, 0, "panel", "panel"), (300, 8, 33, 0, 0, "panel", "panel"), (1000, 16, 7, 5, 1, "panel", "panel"),
         (9, 17, 3, 0, 0, "64", "64"), (64, 64, 32, 0, 0, "64", "64"), (130, 100, 65, 2, 1, "64", "64"),
         (257, 47, 1, 0, 0, "64", "64"), (33, 300, 90, 0, 0, "64", "64"), (20, 1000, 50, 0, 0, "split", "split"),
         (9, 4099, 31, 1, 0, "split", "split"), (700, 515, 301, 6, 3, "split", "split"), (700, 300, 301, 6, 3, "64", "64"), (0, 40, 24, 0, 0, None, None)]


def _gated_inputs(M, K, N, seed=0):
    rng = np.random.default_rng([M, K, N, seed])
    x = rng.standard_normal((M, K)) * np.exp(0.5 * rng.standard_normal((M, 1)))
    return (x, rng.standard_normal((K, 2 * N)) / np.sqrt(K), 0.3 * rng.standard_normal(2 * N),
            1e-3 * rng.standard_normal((M, N)))


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("M,K,N,gap,shift,f32,bf16", GATED)
def test_gated_forward(e3, dt, M, K, N, gap, shift, f32, bf16):  # noqa: F811
    import torch
    x, W, b, _ = _gated_inputs(M, K, N)
    xd, Wd, bd = dev(x, dt, gap, shift), dev(W, dt), dev(b, dt, shift=shift)
    for act, bias in (("silu", True), ("gelu", False), ("relu", True), ("none", False)):
        print("[case] gated_fwd", dt, M, K, N, gap, shift, act, flush=True)
        y, untouched = out_like((M, N), dt, gap, shift)
        names = names_of(e3, lambda: e3.gated_fwd(xd, Wd, bd if bias else None, act, out=y))
        ref, z = ob.gated_fwd(host(xd), host(Wd), host(bd) if bias else None, act)
        assert untouched()
        close(y, ref, dt, act)
        want = f32 if dt == "float32" else bf16
        if want is None:
            assert not names
        else:
            assert any(n.startswith("gated_fwd_" + want) for n in names), names
        got = e3.gated_fwd(xd, Wd, bd if bias else None, act, keep=("z", "z8", "y8"))
        assert torch.equal(got[0], y)                       # the outputs beside y do not change it
        close(got[1], z, dt, "z")
        if M:
            near_steps(got[2][0], z[:, :N])
            near_steps(got[2][1], z[:, N:])
            near_steps(got[3], host(y), share=0.0)


def operand(dz, dt, M, K, N, full=True):
    """dz as the products see it: in bfloat16 but for narrow layers from z in full."""
    return dz if full and K <= 64 and N <= 128 and M * K >= 8 and M * N >= 8 else rounded(dz, dt)


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("M,K,N,gap,shift,f32,bf16", GATED)
@pytest.mark.parametrize("ckpt", [False, True])
def test_gated_backward(e3, dt, M, K, N, gap, shift, f32, bf16, ckpt):  # noqa: F811
    import torch
    x, W, b, dy = _gated_inputs(M, K, N, 1)
    xd, Wd, dyd = dev(x, dt, gap, shift), dev(W, dt), dev(dy, dt, gap, shift)
    for act in ("silu", "gelu", "relu", "none"):
        print("[case] gated_bwd", dt, M, K, N, gap, shift, act, ckpt, flush=True)
        zd = dev(ob.gated_fwd(host(xd), host(Wd), b, act)[1], dt, gap, shift)
        xin, zin, xr, zr = xd, zd, host(xd), host(zd)
        if ckpt and M:
            xin, zin = packed(e3, xr), tuple(packed(e3, v) for v in (zr[:, :N], zr[:, N:]))
            from test_gpu_layers import values
            xr, zr = values(xin), np.concatenate([values(v) for v in zin], 1)
        dx, untouched = out_like((M, K), dt, gap, shift)
        got = e3.gated_bwd(xin, Wd, dyd, zin, act, dx=dx)
        dz = ob.gated_dz(host(dyd), zr, act)
        dzr = operand(dz, dt, M, K, N, not ckpt)
        assert untouched()
        close(got[0], dzr @ host(Wd).T, dt, "dx")
        close(got[1], xr.T @ dzr, dt, "dW")
        close(got[2], dz.sum(0), dt, "db")
        # alone, with the same bits
        for i, k in enumerate(("dx", "dW", "db")):
            alone = e3.gated_bwd(xin if k == "dW" else None, Wd, dyd, zin, act, want=(k,))
            assert torch.equal(alone[i], got[i]) and all(v is None for j, v in enumerate(alone) if j != i)


@pytest.mark.parametrize("act,res,bias,keep", [("none", False, False, ()), ("gelu", False, True, ("z8",)),
                                               ("silu", True, True, ("z", "y8")), ("relu", True, False, ())])
def test_dense_forward_direct(e3, act, res, bias, keep):  # noqa: F811
    """Wide bfloat16 products whose operands go straight to LDS have the bits of those by way of registers,
    which rows of x at odd strides take; rows and columns end inside a tile."""
    import torch
    M, K, N = 16003, 1536, 1000
    g = torch.Generator(device="cuda").manual_seed(17)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, W = normal(M, K), (normal(K, N) / K ** 0.5)
    r, b = (normal(M, N) if res else None), (normal(N) if bias else None)
    odd = torch.zeros(M, K + 3, device="cuda").bfloat16()
    odd[:, :K] = x
    assert names_of(e3, lambda: e3.dense_fwd(x, W, b, r, act, keep)) == {"dense_fwd_256"}
    one, two = (e3.dense_fwd(v, W, b, r, act, keep) for v in (x, odd[:, :K]))
    pairs = zip(one, two) if keep else [(one, two)]
    for u, v in pairs:
        for p, q in ([(u.q, v.q), (u.c, v.c)] if isinstance(u, e3.Packed8) else [(u, v)]):
            assert torch.equal(p, q)
    rows = torch.tensor([0, 1, 255, 256, 8191, M - 20, M - 1], device="cuda")
    z = host(x[rows]) @ host(W) + (host(b) if bias else 0.0)
    y = ol.act(act, z)[0] + (host(r[rows]) if res else 0.0)
    close((one[0] if keep else one)[rows], y, "bfloat16")


@pytest.mark.parametrize("M,K,N", [(16384, 1000, 2048), (8000, 1992, 2112)])
def test_dense_backward_direct(e3, M, K, N):  # noqa: F811
    """The same of dW (x at odd strides), and dx against the definition; the reduction of dW split."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(M)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    x, W, dy, z = normal(M, K), normal(K, N) / K ** 0.5, normal(M, N), normal(M, N)
    odd = torch.zeros(M, K + 3, device="cuda").bfloat16()
    odd[:, :K] = x
    assert {"dense_dz", "dense_bwd_dx_256", "dense_bwd_dw_256"} <= names_of(e3, lambda: e3.dense_bwd(x, W, dy, z, act="silu"))
    one, two = (e3.dense_bwd(v, W, dy, z, act="silu")[:3] for v in (x, odd[:, :K]))
    for u, v in zip(one, two):
        assert torch.equal(u, v)
    zz = host(z)
    dz = host(torch.from_numpy(host(dy) * ol.act("silu", zz)[1]).float().bfloat16())
    rows = [0, 1, 255, 256, M - 20, M - 1]
    close(one[0][rows], dz[rows] @ host(W).T, "bfloat16")
    cols = [0, 1, 255, 256, N - 1]
    close(one[1][:, cols], host(x).T @ dz[:, cols], "bfloat16")


# M, K, N and the kernel, past the sizes above: tiles and row walks
LARGE = [("float32", 262149, 64, 64, 0, "walk"), ("float32", 140000, 32, 128, 0, "walk"), ("float32", 131111, 32, 64, 8, "walk"),
         ("float32", 90001, 64, 192, 0, "walk"), ("float32", 140001, 64, 72, 0, "panel"), ("bfloat16", 262149, 64, 64, 0, "panel"),
         ("float32", 262149, 64, 16, 0, "panel"), ("float32", 131077, 33, 40, 3, "panel"), ("float32", 300007, 8, 64, 0, "panel"),
         ("bfloat16", 262149, 128, 16, 0, "panel"), ("bfloat16", 262176, 64, 32, 0, "panel"), ("bfloat16", 150001, 90, 33, 1, "panel"),
         ("float32", 16403, 100, 300, 0, "128"), ("float32", 4096, 1100, 257, 1, "split_128"), ("bfloat16", 40003, 130, 129, 0, "128"),
         ("bfloat16", 16400, 300, 800, 0, "256"), ("bfloat16", 16400, 320, 800, 0, "256"), ("bfloat16", 16400, 576, 800, 0, "direct"),
         ("bfloat16", 33000, 64, 328, 8, "panel"),
         ("bfloat16", 16387, 192, 1000, 8, "256"), ("bfloat16", 16387, 512, 1000, 8, "direct"), 
         ("bfloat16", 16400, 576, 804, 0, "256"), ("bfloat16", 16400, 576, 800, 4, "256"),
         ("bfloat16", 16400, 320, 804, 0, "256"), ("bfloat16", 16400, 320, 800, 4, "256"), ("bfloat16", 16001, 515, 1021, 6, "256")]


@pytest.mark.parametrize("dt,M,K,N,gap,name", LARGE)
def test_gated_large(e3, dt, M, K, N, gap, name):  # noqa: F811
    """Sampled rows of the forward and of dx, all of db, sampled columns of dW."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(M + K)
    t = getattr(torch, dt)
    wide = torch.randn(M, K + gap, generator=g, device="cuda").to(t)
    x = wide[:, :K]
    W = (torch.randn(K, 2 * N, generator=g, device="cuda") / K ** 0.5).to(t)
    b = (0.1 * torch.randn(2 * N, generator=g, device="cuda")).to(t)
    dy = (1e-3 * torch.randn(M, N, generator=g, device="cuda")).to(t)
    print("[case] gated large", dt, M, K, N, gap, flush=True)
    names = names_of(e3, lambda: e3.gated_fwd(x, W, b))
    assert names == {"gated_fwd_" + name} | ({"gated_fwd_join"} if name.startswith("split") else set())
    y, z, z8, y8 = e3.gated_fwd(x, W, b, keep=("z", "z8", "y8"))
    assert torch.equal(y, e3.gated_fwd(x, W, b))
    rows = np.unique(np.concatenate([np.arange(70), M - 1 - np.arange(70), np.linspace(0, M - 1, 200).astype(int)]))
    pick = torch.from_numpy(rows).cuda()
    ref, zr = ob.gated_fwd(host(x[pick]), host(W), host(b))
    close(y[pick], ref, dt)
    close(z[pick], zr, dt)
    for p, v in ((z8[0], zr[:, :N]), (z8[1], zr[:, N:])):
        near_steps(e3.Packed8(p.q[pick], p.c[pick]), v)
    near_steps(e3.Packed8(y8.q[pick], y8.c[pick]), host(y[pick]), share=0.0)
    dx, dW, db = e3.gated_bwd(x, W, dy, z)
    dz = ob.gated_dz(host(dy), host(z))
    dzr = operand(dz, dt, M, K, N)
    close(dx[pick], dzr[rows] @ host(W).T, dt)
    close(db, dz.sum(0), dt)
    cols = np.unique(np.concatenate([np.arange(min(5, 2 * N)), np.linspace(0, 2 * N - 1, 12).astype(int)]))
    close(dW[:, torch.from_numpy(cols).cuda()], host(x).T @ dzr[:, cols], dt)


@pytest.mark.parametrize("M,K,N", [(16387, 320, 1608), (40003, 256, 520), (8200, 1088, 2056)])
def test_products_past_the_registers_have_the_same_bits(e3, M, K, N):  # noqa: F811
    """Large bfloat16 products whose rows are whole aligned pieces take another way to the same sums."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(M)
    def rows(m, n, gap):
        return torch.empty(m, n + gap, dtype=torch.bfloat16, device="cuda")[:, :n]
    def aligned_and_not(m, n):
        a = torch.randn(m, n, generator=g, device="cuda").bfloat16()
        return a, rows(m, n, 1).copy_(a)
    x, dy = aligned_and_not(M, K), aligned_and_not(M, N)
    W = (torch.randn(K, N, generator=g, device="cuda") / 30).bfloat16()
    b = torch.randn(N, generator=g, device="cuda").bfloat16()
    assert torch.equal(e3.dense_fwd(x[0], W, b, act="gelu"), e3.dense_fwd(x[1], W, b, act="gelu"))
    for u, v in zip(e3.dense_bwd(x[0], W, dy[0]), e3.dense_bwd(x[1], W, dy[1])):
        assert torch.equal(u, v)
    assert torch.equal(e3.gated_fwd(x[0], W), e3.gated_fwd(x[1], W))
    ref = host(dy[0][:64]) @ host(W).T
    close(e3.dense_bwd(None, W, dy[0], want=("dx",))[0][:64], ref, "bfloat16")
    cols = slice(0, N, 61)
    close(e3.dense_bwd(x[0], W, dy[0], want=("dW",))[1][:, cols], host(x[0]).T @ host(dy[0][:, cols]), "bfloat16")


@pytest.mark.parametrize("M,K,N", [(3, 40, 50), (40, 12, 40), (200, 130, 70), (20, 1000, 50), (100000, 64, 40)])
def test_gated_infinities_and_nans_stay_in_their_rows_and_columns(e3, M, K, N):  # noqa: F811
    import torch
    x, W, b, _ = _gated_inputs(M, K, N)
    clean = e3.gated_fwd(dev(x, "float32"), dev(W, "float32"), keep=("z",))[1]
    x[M - 1, 3], x[1, 5] = np.nan, np.inf
    W[2, 7], W[4, N + 9] = np.inf, np.nan
    y, z = e3.gated_fwd(dev(x, "float32"), dev(W, "float32"), keep=("z",))
    rows, cols = [i for i in range(M) if i not in (1, M - 1)], [j for j in range(2 * N) if j not in (7, N + 9)]
    r, c = torch.tensor(rows).cuda(), torch.tensor(cols).cuda()
    assert torch.equal(z[r][:, c], clean[r][:, c])
    assert bool(torch.isnan(z[M - 1]).all()) and not bool(torch.isfinite(z[1]).any())
    assert not bool(torch.isfinite(z[:, 7]).any()) and bool(torch.isnan(z[:, N + 9]).all())
    fine = torch.tensor([j for j in range(N) if j not in (7, 9)]).cuda()
    assert bool(torch.isfinite(y[r][:, fine]).all()) and bool(torch.isnan(y[:, 9]).all())


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12])
def test_gated_float32_range(e3, scale):  # noqa: F811
    x, W, b, _ = _gated_inputs(100, 70, 40)
    xd, Wd = dev(x * scale, "float32"), dev(W, "float32")
    for act in ("relu", "none"):
        y, z = e3.gated_fwd(xd, Wd, act=act, keep=("z",))
        ref, zr = ob.gated_fwd(host(xd), host(Wd), None, act)
        close(z, zr, "float32")
        if scale > 1e-20:
            close(y, ref, "float32")


def test_gated_gradient_equals_differences(e3):  # noqa: F811
    """In float32: z through the kernels, the gradient of <y, dy> along a random direction of x and of W.  Sums of
    800 terms in float32 err by 1e-6 of their size; the difference by its step squared."""
    rng = np.random.default_rng(4)
    x, W, b, _ = _gated_inputs(50, 24, 16)
    dy = rng.standard_normal((50, 16))
    args = [dev(v, "float32") for v in (x, W, b)]
    for act in ("silu", "gelu"):
        z = e3.gated_fwd(*args, act, keep=("z",))[1]
        got = e3.gated_bwd(args[0], args[1], dev(dy, "float32"), z, act)
        for i, g in enumerate(got):
            d = rng.standard_normal(g.shape)
            ends = []
            for sign in (1, -1):
                a = [host(v) for v in args]
                a[i] = a[i] + sign * 1e-4 * d
                ends.append((ob.gated_fwd(*a, act)[0] * dy).sum())
            num = (ends[0] - ends[1]) / 2e-4
            assert abs(num - (host(g) * d).sum()) < 1e-5 * np.linalg.norm(host(g)) * np.sqrt(d.size), (act, i)


# ---------------------------------------------------------------- dropout
@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows,cols,gap,shift", [(1, 1, 0, 0), (3, 7, 0, 1), (5, 8, 0, 0), (2, 9, 3, 0), (33, 515, 6, 5),
                                                 (64, 128, 1920, 0), (700, 1000, 0, 0), (1, 70001, 0, 0), (4099, 3, 0, 0),
                                                 (2, 1 << 20, 0, 0), (0, 40, 0, 0)])
@pytest.mark.parametrize("p,seed,offset", [(0.1, 3, 0), (0.5, (1 << 64) - 1, 1 << 40), (0.0, 5, 1), (1.0, 7, 2),
                                           (0.7303, 0x123456789ABCDEF0, (1 << 64) - 1), (1e-6, 1, 1), (0.999999, 1, 1)])
def test_dropout(e3, dt, rows, cols, gap, shift, p, seed, offset):  # noqa: F811
    """The mask and the kept values are exact: one product in float32, rounded once."""
    import torch
    rng = np.random.default_rng([rows, cols])
    xd, rd = (dev(rng.standard_normal((rows, cols)) + 3, dt, gap, shift) for _ in range(2))
    drop = e3.Dropout(p, seed, offset)
    f = ob.factors(rows, cols, p, seed, offset)
    print("[case] dropout", dt, rows, cols, gap, shift, p, flush=True)
    x32, r32 = host(xd).astype(np.float32), host(rd).astype(np.float32)
    kept = np.where(f > 0, x32 * f.astype(np.float32), np.float32(0))
    for res in (None, rd):
        y, untouched = out_like((rows, cols), dt, gap, shift)
        assert e3.dropout_fwd(xd, drop, res, out=y) is y
        want = torch.from_numpy(kept if res is None else kept + r32).to(getattr(torch, dt))
        assert untouched() and torch.equal(y.cpu(), want)
    dx, untouched = out_like((rows, cols), dt, gap, shift)
    e3.dropout_bwd(xd, drop, dx=dx)
    assert untouched() and torch.equal(dx.cpu(), torch.from_numpy(kept).to(getattr(torch, dt)))
    # in place
    if rows:
        for target, res in ((xd, None), (rd, rd), (xd, rd)):
            want = e3.dropout_fwd(xd, drop, res)
            into = target.clone()
            got = e3.dropout_fwd(into if target is xd else xd, drop, None if res is None else into if target is rd else rd,
                                 out=into)
            assert torch.equal(got, want)


def test_dropped_values_are_not_looked_at(e3):  # noqa: F811
    import torch
    x = torch.full((50, 300), float("nan"), device="cuda")
    keep = torch.from_numpy(ob.kept(50, 300, 0.4, 9, 2)).cuda()
    x[keep] = 1.0
    for dt in DTS:
        y = e3.dropout_fwd(x.to(getattr(torch, dt)), e3.Dropout(0.4, 9, 2))
        assert bool((y[~keep] == 0).all()) and bool((y[keep] > 1.6).all())


def test_dropout_far_rows(e3):  # noqa: F811
    """Rows past 2^32, and rows whose offsets pass 32 bits."""
    import torch
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    drop = e3.Dropout(0.5, 77, 3)
    rows = (1 << 32) + 70
    x = torch.ones(rows, 1, dtype=torch.bfloat16, device="cuda")
    y = e3.dropout_fwd(x, drop)
    at = np.concatenate([np.arange(60), np.arange((1 << 32) - 30, rows)])
    want = ob.kept(at, 1, 0.5, 77, 3)
    assert np.array_equal(host(y[torch.from_numpy(at).cuda()]) > 0, want)
    del x, y
    ld = (1 << 31) + 11
    wide = torch.empty(5 * ld, dtype=torch.bfloat16, device="cuda")
    x = wide[:5 * ld].view(5, ld)[:, :100]
    x.fill_(1.0)
    assert np.array_equal(host(e3.dropout_fwd(x, drop)) > 0, ob.kept(5, 100, 0.5, 77, 3))
    s, y = e3.residual_norm_fwd(x, x, pre=(None, None), drop=drop)
    assert np.array_equal(host(s) > 2, ob.kept(5, 100, 0.5, 77, 3))


# ---------------------------------------------------------------- residual norms
# rows, cols, gap, shift
SIZES = [(1, 1, 0, 0), (3, 2, 0, 0), (2, 7, 1, 1), (70, 16, 0, 0), (33, 31, 0, 0), (64, 32, 4, 0), (50, 65, 0, 3),
         (129, 128, 1920, 0), (5003, 64, 0, 0), (40, 256, 0, 0), (10, 515, 0, 0), (9, 1000, 24, 8), (700, 1025, 0, 0),
         (5, 2047, 1, 0), (4, 2049, 0, 0), (6, 4100, 0, 2), (3, 8192, 0, 0), (3, 8193, 5, 0), (2, 16385, 0, 1),
         (2, 40001, 0, 0), (0, 40, 0, 0)]
# norm, after, before, gate, p, weights, residual
KINDS = [("rms", True, True, "row", 0.1, True, True), ("layer", True, True, "full", 0.3, True, True),
         ("rms", False, True, "none", 0.0, True, True), ("layer", False, True, "row", 0.0, True, True),
         ("rms", True, False, "full", 0.5, False, True), ("layer", True, False, "none", 0.0, True, False),
         ("layer", True, True, "none", 0.0, False, True), ("rms", False, False, "row", 0.2, True, True),
         ("layer", False, True, "full", 0.2, False, True), ("rms", True, True, "none", 0.0, True, False)]


def _residual_inputs(rows, cols, norm, after, before, gate, weights, seed=0):
    rng = np.random.default_rng([rows, cols, seed])
    h = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1))) + 0.5
    r, ds, dy = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))
    g = {"none": None, "row": 0.5 + 0.3 * rng.standard_normal(cols), "full": rng.random((rows, cols))}[gate]
    w = []
    for there in (after, before):
        pair = (1 + 0.3 * rng.standard_normal(cols), rng.standard_normal(cols) if norm == "layer" else None)
        w.append((pair if weights else (None, None)) if there else None)
    return h, r, g, w[0], w[1], 1e-3 * ds, 1e-3 * dy


def _pair(w, dt, shift):
    return None if w is None else tuple(None if v is None else dev(v, dt, shift=shift) for v in w)


def _host_pair(w):
    return None if w is None else tuple(None if v is None else host(v) for v in w)


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("rows,cols,gap,shift", SIZES)
@pytest.mark.parametrize("norm,after,before,gate,p,weights,res", KINDS)
def test_residual_norm(e3, dt, rows, cols, gap, shift, norm, after, before, gate, p, weights, res):  # noqa: F811
    import torch
    h, r, g, post, pre, ds, dy = _residual_inputs(rows, cols, norm, after, before, gate, weights)
    hd, rd, dsd, dyd = (dev(v, dt, gap, shift) for v in (h, r, ds, dy))
    gd = None if g is None else dev(g, dt, gap if gate == "full" else 0, shift)
    post, pre = _pair(post, dt, shift), _pair(pre, dt, shift)
    drop = e3.Dropout(p, 21, 4) if p else None
    f = ob.factors(rows, cols, p, 21, 4) if p else None
    scale = 0.75
    print("[case] residual_norm", dt, rows, cols, gap, shift, norm, after, before, gate, p, flush=True)
    s, untouched = out_like((rows, cols), dt, gap, shift)
    y, untouched_y = out_like((rows, cols), dt, gap, shift)
    got = e3.residual_norm_fwd(hd, rd if res else None, gd, scale, norm, post, pre, 1e-5, drop, keep=("stats",), out=s,
                               y=y if before else None)
    stats = got[-1]
    assert untouched() and untouched_y() and len(got) == 2 + before
    assert stats.shape == ((1 + (norm == "layer")) * (after + before), rows)
    hr, gr, pr, qr = host(hd), None if g is None else host(gd), _host_pair(post), _host_pair(pre)
    ref_s, ref_y, first, last = ob.residual_norm_fwd(hr, host(rd) if res else None, gr, scale, norm, pr, qr, 1e-5, f)
    if rows == 0:
        if before:
            assert e3.residual_norm_bwd(hd, s, stats, dyd, dsd, gd, scale, norm, post, pre, drop)[0].shape == (0, cols)
        return
    # one column: a layer norm's deviations are 0, and so are y's terms but beta
    tiny = cols == 1 and norm == "layer"
    close(s, ref_s, dt, "s")
    if before and not tiny:
        close(y, ref_y, dt, "y")
    want = [v for st in (first, last) if st is not None for v in st if v is not None]
    k = 0
    for st in (first, last):
        if st is None:
            continue
        if norm == "layer":
            # Each of a row's values x carries roundings of 2^-24 |x| with it, so that their mean is off by up to
            # 2^-24 mean |x| < 2^-24 (|mean| + 1 / rstd) per rounding, however small it is itself: 16,385 values
            # of size 1 with a mean of 0.0018 give it to 1.5e-8, 8.6e-6 of it.
            assert (np.abs(host(stats[k]) - st[0]) < 4e-6 * (np.abs(st[0]) + 1 / st[1])).all(), k
            k += 1
        if not tiny:
            assert rel_l2(stats[k].cpu(), st[1]) < 4e-6, k
        k += 1
    # fewer outputs, and s in place of r: the same bits
    again = e3.residual_norm_fwd(hd, rd if res else None, gd, scale, norm, post, pre, 1e-5, drop)
    if before:
        assert torch.equal(again[0], s) and torch.equal(again[1], y)
    else:
        assert torch.equal(again, s)
    if res:
        over = rd.clone()
        again = e3.residual_norm_fwd(hd, over, gd, scale, norm, post, pre, 1e-5, drop, out=over)
        assert torch.equal(over, s) and (not before or torch.equal(again[1], y))

    # backward, from the stored s and the oracle's statistics
    sd = dev(ref_s, dt, gap, shift)
    st32 = torch.from_numpy(np.stack(want).astype(np.float32)).cuda() if want else None
    given = iter([] if st32 is None else host(st32))
    first, last = (None if st is None else tuple(None if v is None else next(given) for v in st) for st in (first, last))
    dr, untouched = out_like((rows, cols), dt, gap, shift)
    dh, untouched_h = out_like((rows, cols), dt, gap, shift)
    got = e3.residual_norm_bwd(hd, sd, st32, dyd if before else None, dsd, gd, scale, norm, post, pre, drop, dres=dr, dh=dh)
    ref = ob.residual_norm_bwd(hr, host(sd), first, last, host(dyd) if before else None, host(dsd), gr, scale, norm, pr, qr, f)
    assert untouched() and untouched_h()
    if tiny:
        return
    close(dr, ref[0], dt, "dres")
    if not (cols <= 2 and after):       # (a norm of one or two columns cancels nearly all of its cotangent)
        close(dh, ref[1], dt, "dh")
    if g is not None:
        close(got[2], ref[2], dt, "dgate")
    else:
        assert got[2] is None
    for k, w in ((3, post), (4, pre)):
        assert (got[k] is None) == (w is None)
        if w is not None:
            for a, b, c in zip(got[k], ref[k], w):
                assert (a is None) == (c is None)
                if a is not None:
                    close(a, b, dt, ("dpost", "dpre")[k - 3])
    # one gradient at a time: the same bits
    for i, k in enumerate(("dres", "dh", "dgate", "dpost", "dpre")):
        alone = e3.residual_norm_bwd(hd, sd, st32, dyd if before else None, dsd, gd, scale, norm, post, pre, drop, want=(k,))
        for j, v in enumerate(alone):
            if j != i:
                assert v is None
            elif isinstance(v, tuple):
                assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(v, got[i]))
            else:
                assert (v is None and got[i] is None) or torch.equal(v, got[i])


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", [64, 1024, 20000])
def test_residual_norm_without_ds(e3, dt, cols):  # noqa: F811
    """ds None is a ds of zeros."""
    import torch
    h, r, g, post, pre, ds, dy = _residual_inputs(9, cols, "rms", True, True, "row", True)
    hd, rd, dyd, gd = dev(h, dt), dev(r, dt), dev(dy, dt), dev(g, dt)
    post, pre = _pair(post, dt, 0), _pair(pre, dt, 0)
    s, y, st = e3.residual_norm_fwd(hd, rd, gd, 0.5, "rms", post, pre, keep=("stats",))
    a = e3.residual_norm_bwd(hd, s, st, dyd, None, gd, 0.5, "rms", post, pre)
    b = e3.residual_norm_bwd(hd, s, st, dyd, torch.zeros_like(dyd), gd, 0.5, "rms", post, pre)
    for u, v in zip(a, b):
        u, v = (u[0], v[0]) if isinstance(u, tuple) else (u, v)
        assert torch.equal(u, v)


@pytest.mark.parametrize("cols", [7, 64, 256, 700, 1025, 4100, 8192, 20000])
def test_residual_norm_of_a_large_mean(e3, cols):  # noqa: F811
    """The mean's rounding to float32 stays out of y (a mean 3,000 times the deviation would move it by 2e-4)."""
    rng = np.random.default_rng(cols)
    h = dev(3000 + rng.standard_normal((40, cols)), "float32")
    for kw in ({"post": (None, None)}, {"pre": (None, None)}):
        out = e3.residual_norm_fwd(h, norm="layer", **kw)
        ref = ob.residual_norm_fwd(host(h), norm="layer", **kw)
        close(out if "post" in kw else out[1], ref[0] if "post" in kw else ref[1], "float32")


@pytest.mark.parametrize("cols", [24, 700, 3001, 20000])
def test_residual_norm_bad_rows_stay_alone(e3, cols):  # noqa: F811
    import torch
    h, r, g, post, pre, ds, dy = _residual_inputs(30, cols, "layer", True, True, "full", True)
    args = [dev(v, "float32") for v in (h, r, g)]
    post, pre = _pair(post, "float32", 0), _pair(pre, "float32", 0)
    clean = e3.residual_norm_fwd(*args, 1.0, "layer", post, pre)
    args[0][3, cols - 1], args[1][7, 2], args[2][11, 5], args[0][13, 1] = (float("nan"), float("inf"), float("nan"), float("inf"))
    got = e3.residual_norm_fwd(*args, 1.0, "layer", post, pre)
    fine = torch.tensor([i for i in range(30) if i not in (3, 7, 11, 13)]).cuda()
    for a, b in zip(clean, got):
        assert torch.equal(a[fine], b[fine])
    assert bool(torch.isnan(got[1][torch.tensor([3, 7, 11, 13]).cuda()]).all())
    # a row of zeros: rstd = 1 / sqrt(eps), y = beta
    zero = torch.zeros(4, cols, device="cuda")
    s, y, st = e3.residual_norm_fwd(zero, zero, norm="rms", pre=(None, None), keep=("stats",))
    assert not bool(s.any()) and not bool(y.any()) and np.allclose(host(st), 1e-5 ** -0.5)


@pytest.mark.parametrize("dt,rows,cols,norm,gate", [("bfloat16", 20001, 1024, "rms", "row"), ("bfloat16", 300001, 64, "layer", "row"),
                                                   ("float32", 20001, 515, "layer", "full"), ("float32", 9001, 1024, "rms", "full"),
                                                   ("bfloat16", 5001, 4096, "layer", "none"), ("float32", 40001, 256, "rms", "none"),
                                                   ("bfloat16", 2001, 10001, "rms", "row")])
def test_residual_norm_many_rows(e3, dt, rows, cols, norm, gate):  # noqa: F811
    """Sums over many rows, and outputs past the caches."""
    import torch
    h, r, g, post, pre, ds, dy = _residual_inputs(rows, cols, norm, True, True, gate, True)
    hd, rd, dsd, dyd = (dev(v, dt) for v in (h, r, ds, dy))
    gd = None if g is None else dev(g, dt)
    post, pre = _pair(post, dt, 0), _pair(pre, dt, 0)
    drop, f = e3.Dropout(0.2, 5), ob.factors(rows, cols, 0.2, 5)
    print("[case] residual_norm many", dt, rows, cols, norm, gate, flush=True)
    s, y, st = e3.residual_norm_fwd(hd, rd, gd, 1.0, norm, post, pre, 1e-5, drop, keep=("stats",))
    gr, pr, qr = None if g is None else host(gd), _host_pair(post), _host_pair(pre)
    ref_s, ref_y, first, last = ob.residual_norm_fwd(host(hd), host(rd), gr, 1.0, norm, pr, qr, 1e-5, f)
    close(s, ref_s, dt, "s")
    close(y, ref_y, dt, "y")
    given = iter(host(st))
    first, last = (tuple(None if v is None else next(given) for v in x) for x in (first, last))
    got = e3.residual_norm_bwd(hd, s, st, dyd, dsd, gd, 1.0, norm, post, pre, drop)
    ref = ob.residual_norm_bwd(host(hd), host(s), first, last, host(dyd), host(dsd), gr, 1.0, norm, pr, qr, f)
    for name, a, b in zip(("dres", "dh", "dgate", "dpost", "dpre"), got, ref):
        for u, v in zip(a, b) if isinstance(a, tuple) else ((a, b),):
            if u is not None:
                close(u, v, dt, name)
    again = e3.residual_norm_bwd(hd, s, st, dyd, dsd, gd, 1.0, norm, post, pre, drop)
    for a, b in zip(got, again):
        for u, v in zip(a, b) if isinstance(a, tuple) else ((a, b),):
            assert u is None or torch.equal(u, v)


def test_residual_norm_gradient_equals_differences(e3):  # noqa: F811
    rng = np.random.default_rng(6)
    h, r, g, post, pre, _, _ = _residual_inputs(20, 48, "layer", True, True, "row", True)
    ds, dy = rng.standard_normal((2, 20, 48))
    f = ob.factors(20, 48, 0.25, 8)
    names = [h, r, g, *post, *pre]
    d = [dev(v, "float32") for v in names]
    s, y, st = e3.residual_norm_fwd(*d[:3], 0.5, "layer", tuple(d[3:5]), tuple(d[5:]), 1e-5, e3.Dropout(0.25, 8), keep=("stats",))
    dr, dh, dg, dpost, dpre = e3.residual_norm_bwd(d[0], s, st, dev(dy, "float32"), dev(ds, "float32"), d[2], 0.5, "layer",
                                                   tuple(d[3:5]), tuple(d[5:]), e3.Dropout(0.25, 8))
    for i, got in enumerate((dh, dr, dg, *dpost, *dpre)):
        step = rng.standard_normal(names[i].shape)
        ends = []
        for sign in (1, -1):
            a = list(names)
            a[i] = names[i] + sign * 1e-4 * step
            u, v, _, _ = ob.residual_norm_fwd(*a[:3], 0.5, "layer", tuple(a[3:5]), tuple(a[5:]), 1e-5, f)
            ends.append((u * ds).sum() + (v * dy).sum())
        num = (ends[0] - ends[1]) / 2e-4
        assert abs(num - (host(got) * step).sum()) < 1e-5 * np.linalg.norm(host(got)) * np.sqrt(step.size), i


@pytest.mark.parametrize("M,K,N", [(17_000_003, 8, 64), (9_000_007, 8, 130)])
def test_gated_past_two_billion_values(e3, M, K, N):  # noqa: F811
    """z (and dz, where it is written) has more than 2^31 values: rows of both ends."""
    import torch
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(M, K, generator=g, device="cuda").bfloat16()
    W = torch.randn(K, 2 * N, generator=g, device="cuda").bfloat16()
    dy = torch.randn(M, N, generator=g, device="cuda").bfloat16()
    print("[case] gated large", M, K, N, flush=True)
    y, z = e3.gated_fwd(x, W, keep=("z",))
    dx = e3.gated_bwd(None, W, dy, z, want=("dx",))[0]
    rows = torch.cat([torch.arange(100), torch.arange(M - 100, M), torch.arange((1 << 31) // (2 * N) - 50, (1 << 31) // (2 * N) + 50)]).cuda()
    ref, zr = ob.gated_fwd(host(x[rows]), host(W))
    close(y[rows], ref, "bfloat16")
    close(z[rows], zr, "bfloat16")
    dz = operand(ob.gated_dz(host(dy[rows]), host(z[rows])), "bfloat16", M, K, N)
    close(dx[rows], dz @ host(W).T, "bfloat16")
    # the sums over rows: those of the last rows alone reach dW and db
    dy[:-100] = 0
    dW, db = e3.gated_bwd(x, W, dy, z, want=("dW", "db"))[1:]
    last = torch.arange(M - 100, M).cuda()
    dz = ob.gated_dz(host(dy[last]), host(z[last]))
    close(dW, host(x[last]).T @ operand(dz, "bfloat16", M, K, N), "bfloat16")
    close(db, dz.sum(0), "bfloat16")


def test_residual_norm_past_two_billion_values(e3):  # noqa: F811
    import torch
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    M, K = 2_100_007, 1024
    g = torch.Generator(device="cuda").manual_seed(2)
    h, r, dy, ds = (torch.randn(M, K, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    w = ((1 + 0.2 * torch.randn(K, generator=g, device="cuda")).bfloat16(), None)
    drop = e3.Dropout(0.3, 5, 9)
    print("[case] residual_norm large", M, K, flush=True)
    s, y, st = e3.residual_norm_fwd(h, r, None, 0.5, "rms", w, w, drop=drop, keep=("stats",))
    dr, dh, _, _, _ = e3.residual_norm_bwd(h, s, st, dy, ds, None, 0.5, "rms", w, w, drop, want=("dres", "dh"))
    rows = np.concatenate([np.arange(40), np.arange((1 << 31) // K - 20, (1 << 31) // K + 20), np.arange(M - 40, M)])
    pick = torch.from_numpy(rows).cuda()
    wh, f = (host(w[0]), None), ob.factors(rows, K, 0.3, 5, 9)
    rs, ry, first, last = ob.residual_norm_fwd(host(h[pick]), host(r[pick]), None, 0.5, "rms", wh, wh, 1e-5, f)
    close(s[pick], rs, "bfloat16")
    close(y[pick], ry, "bfloat16")
    got = host(st[:, pick])
    ref = ob.residual_norm_bwd(host(h[pick]), host(s[pick]), (None, got[0]), (None, got[1]), host(dy[pick]), host(ds[pick]), None,
                               0.5, "rms", wh, wh, f)
    close(dr[pick], ref[0], "bfloat16")
    close(dh[pick], ref[1], "bfloat16")


@pytest.mark.parametrize("M,K,N", [(1000, 64, 128), (700, 24, 20), (40, 64, 33), (900, 100, 60)])
def test_gated_backward_bad_values_stay_in_their_rows_and_columns(e3, M, K, N):  # noqa: F811
    """float32: an infinity in x reaches its row of dW, a NaN in dy its row of dx and its columns of dW and db."""
    import torch
    x, W, b, dy = _gated_inputs(M, K, N)
    z = ob.gated_fwd(x, W, b)[1]
    x[M // 2, 3], dy[M - 1, 5] = np.inf, np.nan
    dx, dW, db = e3.gated_bwd(dev(x, "float32"), dev(W, "float32"), dev(dy, "float32"), dev(z, "float32"))
    clean = dy.copy()
    clean[M - 1, 5] = 0
    dz = ob.gated_dz(clean, z)
    rows = [i for i in range(M) if i != M - 1]
    close(dx[torch.tensor(rows).cuda()], dz[rows] @ W.T, "float32")
    assert bool(torch.isnan(dx[M - 1]).all())
    ks, js = [k for k in range(K) if k != 3], [j for j in range(2 * N) if j not in (5, N + 5)]
    close(dW[torch.tensor(ks).cuda()][:, torch.tensor(js).cuda()], (x[:, ks].T @ dz)[:, js], "float32")
    assert not bool(torch.isfinite(dW[3]).any()) and bool(torch.isnan(dW[:, 5]).all()) and bool(torch.isnan(dW[:, N + 5]).all())
    close(db[torch.tensor(js).cuda()], dz.sum(0)[js], "float32")
    assert bool(torch.isnan(db[5])) and bool(torch.isnan(db[N + 5]))


@pytest.mark.parametrize("scale", [1e-30, 1e12, 1e18])
@pytest.mark.parametrize("M,K,N", [(500, 64, 100), (500, 70, 100)])
def test_gated_backward_float32_range(e3, scale, M, K, N):  # noqa: F811
    """Operands whose scaled terms or sums leave the matrix cores' range."""
    x, W, b, dy = _gated_inputs(M, K, N)
    xd, Wd, zd, dyd = dev(x * scale, "float32"), dev(W, "float32"), dev(ob.gated_fwd(x, W, b)[1], "float32"), dev(dy, "float32")
    dz = ob.gated_dz(host(dyd), host(zd))
    dx, dW, db = e3.gated_bwd(xd, Wd, dyd, zd)
    close(dx, dz @ host(Wd).T, "float32")
    close(dW, host(xd).T @ dz, "float32")
    dx = e3.gated_bwd(None, Wd, dev(dy * scale, "float32"), zd, want=("dx",))[0]
    close(dx, ob.gated_dz(host(dev(dy * scale, "float32")), host(zd)) @ host(Wd).T, "float32")


# ---------------------------------------------------------------- as they are used
def _block(e3, dt, packs, M=900, D=96, F=160):  # noqa: F811
    """Two residual blocks, forward and backward call by call, against float64 automatic differentiation."""
    import torch
    t = getattr(torch, dt)
    g = torch.Generator().manual_seed(3)
    def rand(*shape, scale=1.0):
        return (scale * torch.randn(*shape, generator=g)).to(t).cuda()
    x, dout = rand(M, D), rand(M, D)
    P = [{"g1": 1 + rand(D, scale=0.1), "W1": rand(D, 2 * F, scale=D ** -0.5), "b1": rand(2 * F, scale=0.1),
          "W2": rand(F, D, scale=F ** -0.5), "gate": rand(D, scale=0.3) + 0.5, "g2": 1 + rand(D, scale=0.1)} for _ in range(2)]
    drops = [e3.Dropout(0.2, 17, k) for k in range(2)]
    s, y, st = e3.residual_norm_fwd(x, pre=(P[0]["g1"], None), keep=("stats",))
    kept = [(x, s, st)]
    acts = []
    for k, p in enumerate(P):
        if packs:
            y8 = e3.pack8(y)
            a, z, a8 = e3.gated_fwd(y, p["W1"], p["b1"], keep=("z8", "y8"))
        else:
            a, z = e3.gated_fwd(y, p["W1"], p["b1"], keep=("z",))
            y8, a8 = y, a
        h = e3.dense_fwd(a, p["W2"])
        acts.append((y8, z, a8))
        nxt = (P[k + 1]["g1"], None) if k == 0 else None
        out = e3.residual_norm_fwd(h, s, p["gate"], 0.7, "rms", (p["g2"], None), nxt, drop=drops[k], keep=("stats",))
        s, st = out[0], out[-1]
        y = out[1] if k == 0 else None
        kept.append((h, s, st))
    # backward
    grads = [{}, {}]
    ds, dy = dout, None
    for k in (1, 0):
        p = P[k]
        nxt = (P[k + 1]["g1"], None) if k == 0 else None
        h, s_k, st = kept[k + 1]
        ds, dh, grads[k]["gate"], (grads[k]["g2"], _), dpre = e3.residual_norm_bwd(
            h, s_k, st, dy, ds, p["gate"], 0.7, "rms", (p["g2"], None), nxt, drops[k])
        if k == 0:
            grads[1]["g1"] = dpre[0]
        y8, z, a8 = acts[k]
        da, grads[k]["W2"], _ = e3.dense_bwd(a8, p["W2"], dh, want=("dx", "dW"))
        dy, grads[k]["W1"], grads[k]["b1"] = e3.gated_bwd(y8, p["W1"], da, z)
    h, s_0, st = kept[0]
    dx, _, _, _, (grads[0]["g1"], _) = e3.residual_norm_bwd(None, s_0, st, dy, ds, pre=(P[0]["g1"], None), want=("dres", "dpre"))

    # the reference
    Q = [{k: v.double().cpu().requires_grad_() for k, v in p.items()} for p in P]
    x64 = x.double().cpu().requires_grad_()
    def rms(v, w):
        return v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5) * w
    s64 = x64
    for k, q in enumerate(Q):
        z64 = rms(s64, q["g1"]) @ q["W1"] + q["b1"]
        h64 = (torch.nn.functional.silu(z64[:, :F]) * z64[:, F:]) @ q["W2"]
        s64 = s64 + 0.7 * q["gate"] * torch.from_numpy(ob.factors(M, D, 0.2, 17, k)) * rms(h64, q["g2"])
    (s64 * dout.double().cpu()).sum().backward()
    out = [(s, s64.detach()), (dx, x64.grad)]
    for k in range(2):
        out += [(grads[k][n], Q[k][n].grad) for n in Q[k]]
    return [float((a.double().cpu() - b).norm() / b.norm()) for a, b in out]


@pytest.mark.parametrize("dt,packs,bar", [("float32", False, 2e-5), ("float32", True, 0.05), ("bfloat16", False, 0.05)])
def test_two_blocks_together(e3, dt, packs, bar):  # noqa: F811
    """float32: 20 operators in a row, 1e-6 each.  From 8 bits each saved value is off by up to 1/127 of its
    group's largest; bfloat16 rounds each activation and gradient by 2^-9, some 20 times and with gains of a few."""
    errors = _block(e3, dt, packs)
    print(errors, flush=True)
    assert max(errors) < bar
    assert errors[0] < (2e-5 if dt == "float32" else bar)


# ---------------------------------------------------------------- how calls are made
def test_repeats_are_bitwise_equal(e3):  # noqa: F811
    import torch
    x, W, b, dy = (dev(v, "bfloat16") for v in _gated_inputs(3000, 200, 150))
    y, z = e3.gated_fwd(x, W, b, keep=("z",))
    for _ in range(3):
        assert torch.equal(e3.gated_fwd(x, W, b), y)
        for a, c in zip(e3.gated_bwd(x, W, dy, z), e3.gated_bwd(x, W, dy, z)):
            assert torch.equal(a, c)


def test_on_another_stream(e3):  # noqa: F811
    """Inputs made on a stream are used on it; outputs and scratch belong to it."""
    import torch
    side = torch.cuda.Stream()
    x, W, b, dy = _gated_inputs(2000, 300, 200)
    ref = e3.gated_fwd(dev(x, "float32"), dev(W, "float32"), keep=("z",))
    refs = e3.gated_bwd(dev(x, "float32"), dev(W, "float32"), dev(dy, "float32"), ref[1])
    drop = e3.Dropout(0.3, 4)
    rs = e3.residual_norm_fwd(ref[0], ref[0], pre=(None, None), drop=drop)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        xs, Ws, dys = dev(x, "float32"), dev(W, "float32"), dev(dy, "float32")
    got = e3.gated_fwd(xs, Ws, keep=("z",), stream=side)
    grads = e3.gated_bwd(xs, Ws, dys, got[1], stream=side)
    out = e3.residual_norm_fwd(got[0], got[0], pre=(None, None), drop=drop, stream=side)
    d = e3.dropout_bwd(e3.dropout_fwd(got[0], drop, stream=side), drop, stream=side)
    side.synchronize()
    for a, c in zip((*got, *grads, *out), (*ref, *refs, *rs)):
        assert torch.equal(a, c)
    assert torch.equal(d, e3.dropout_bwd(e3.dropout_fwd(ref[0], drop), drop))


def test_in_a_captured_graph(e3):  # noqa: F811
    """A training pass, replayed with new inputs and a counter counted up in between: each replay is the eager
    pass on what is there then.  Two graphs with scratch of their own, eager work between replays."""
    import torch
    x, W, b, dy = (dev(v, "float32") for v in _gated_inputs(700, 96, 96, 2))
    W2 = dev(np.random.default_rng(0).standard_normal((96, 96)) / 10, "float32")
    gamma = dev(1 + 0.1 * np.random.default_rng(1).standard_normal(96), "float32")
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(counter):
        drop = e3.Dropout(0.25, 99, 1 << 33, counter)
        y, z = e3.gated_fwd(x, W, b, keep=("z",))
        h = e3.dense_fwd(y, W2)
        s, n, st = e3.residual_norm_fwd(h, x, gamma, 0.5, "rms", (gamma, None), (gamma, None), drop=drop, keep=("stats",))
        ds, dh, dgate, dpost, dpre = e3.residual_norm_bwd(h, s, st, dy, dy, gamma, 0.5, "rms", (gamma, None), (gamma, None), drop)
        da, dW2, _ = e3.dense_bwd(y, W2, dh, want=("dx", "dW"))
        dx, dW, db = e3.gated_bwd(x, W, da, z)
        e = e3.dropout_bwd(e3.dropout_fwd(x, drop, s), drop)
        return s, n, ds, dgate, dpost[0], dpre[0], dW2, dx, dW, db, e
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for _ in range(2):
            step(counter)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                outs = step(counter)
            graphs.append((graph, outs))
    torch.cuda.current_stream().wait_stream(side)
    seen = []
    for k in range(4):
        x.copy_(dev(_gated_inputs(700, 96, 96, 10 + k)[0], "float32"))
        counter.fill_(3 * k)
        want = [v.clone() for v in step(counter)]
        for graph, outs in graphs:
            graph.replay()
            torch.cuda.synchronize()
            for i, (a, c) in enumerate(zip(outs, want)):
                assert torch.equal(a, c), (k, i)
        fixed = e3.dropout_fwd(x, e3.Dropout(0.25, 99, (1 << 33) + 3 * k))
        assert torch.equal(fixed, e3.dropout_fwd(x, e3.Dropout(0.25, 99, 1 << 33, counter)))
        seen.append(fixed != 0)
    assert not torch.equal(seen[0], seen[1])


def test_refusals(e3):  # noqa: F811
    import torch
    x, W, b, dy = (dev(v, "float32") for v in _gated_inputs(20, 24, 16))
    z = e3.gated_fwd(x, W, keep=("z",))[1]
    drop = e3.Dropout(0.5, 1)
    bad = [
        (ValueError, lambda: e3.gated_fwd(x, W[:, :31].contiguous())),
        (ValueError, lambda: e3.gated_fwd(x, W[:23].contiguous())),
        (ValueError, lambda: e3.gated_fwd(x, W, b[:30].contiguous())),
        (ValueError, lambda: e3.gated_fwd(x, W, act="tanh")),
        (ValueError, lambda: e3.gated_fwd(x, W, keep=("g",))),
        (ValueError, lambda: e3.gated_fwd(x.cpu(), W)),
        (ValueError, lambda: e3.gated_fwd(x, W.t())),
        (TypeError, lambda: e3.gated_fwd(x, W.bfloat16())),
        (TypeError, lambda: e3.gated_fwd(x.double(), W)),
        (TypeError, lambda: e3.gated_fwd([1.0], W)),
        (ValueError, lambda: e3.gated_fwd(x, W, out=torch.empty(20, 15, device="cuda"))),
        (ValueError, lambda: e3.gated_bwd(x, W, dy, z[:, :16])),
        (ValueError, lambda: e3.gated_bwd(x, W, dy, (e3.pack8(dy),))),
        (TypeError, lambda: e3.gated_bwd(x, W, dy, (z, z))),
        (TypeError, lambda: e3.gated_bwd(x, W, dy, None)),
        (e3.E3Error, lambda: e3.gated_bwd(None, W, dy, z)),
        (ValueError, lambda: e3.Dropout(1.5, 0)),
        (ValueError, lambda: e3.Dropout(float("nan"), 0)),
        (ValueError, lambda: e3.Dropout(0.5, -1)),
        (ValueError, lambda: e3.Dropout(0.5, 1 << 64)),
        (ValueError, lambda: e3.Dropout(0.5, 0, 1 << 64)),
        (TypeError, lambda: e3.dropout_fwd(x, 0.5)),
        (TypeError, lambda: e3.dropout_bwd(x, None)),
        (TypeError, lambda: e3.dropout_fwd(x, e3.Dropout(0.5, 1, 0, torch.zeros(1, device="cuda")))),
        (ValueError, lambda: e3.dropout_fwd(x, e3.Dropout(0.5, 1, 0, torch.zeros(1, dtype=torch.int64)))),
        (ValueError, lambda: e3.dropout_fwd(x, e3.Dropout(0.5, 1, 0, torch.zeros(2, dtype=torch.int64, device="cuda")))),
        (ValueError, lambda: e3.dropout_fwd(x, drop, x[:10])),
        (ValueError, lambda: e3.dropout_fwd(x[0], drop)),
        (ValueError, lambda: e3.residual_norm_fwd(x, norm="batch", pre=(None, None))),
        (ValueError, lambda: e3.residual_norm_fwd(x, norm="rms", pre=(None, b[:24].contiguous()))),
        (TypeError, lambda: e3.residual_norm_fwd(x, pre=b[:24])),
        (ValueError, lambda: e3.residual_norm_fwd(x, pre=(b[:23].contiguous(), None))),
        (ValueError, lambda: e3.residual_norm_fwd(x, post=(None, None), y=x)),
        (ValueError, lambda: e3.residual_norm_fwd(x, gate=b[:20].contiguous())),
        (ValueError, lambda: e3.residual_norm_fwd(x, gate=x.new_ones(1, 24).expand(20, 24))),
        (TypeError, lambda: e3.residual_norm_fwd(x, pre=(None, None), drop=0.1)),
        (ValueError, lambda: e3.residual_norm_fwd(x, keep=("mean",))),
        (ValueError, lambda: e3.residual_norm_bwd(x, x, None)),
        (ValueError, lambda: e3.residual_norm_bwd(x, x, None, dy=x)),
        (ValueError, lambda: e3.residual_norm_bwd(x, x, None, ds=x, pre=(None, None))),
        (ValueError, lambda: e3.residual_norm_bwd(x, x, torch.empty(2, 20, device="cuda"), dy=x, pre=(None, None))),
        (e3.E3Error, lambda: e3.residual_norm_bwd(None, x, torch.empty(1, 20, device="cuda"), ds=x, post=(None, None))),
        (e3.E3Error, lambda: e3.residual_norm_bwd(x, None, torch.empty(1, 20, device="cuda"), dy=x, pre=(None, None))),
    ]
    for k, (kind, call) in enumerate(bad):
        with pytest.raises(kind):
            call()
            pytest.fail(f"call {k} was not refused")


def test_scratch_is_checked(e3):  # noqa: F811
    import torch
    x, W, b, dy = (dev(v, "float32") for v in _gated_inputs(16, 1000, 250))
    z = e3.gated_fwd(x, W, keep=("z",))[1]
    f, bw = e3.gated_workspace_size(16, 1000, 250)
    rn = e3.residual_norm_workspace_size(16, 250)
    st = torch.ones(1, 16, device="cuda")
    calls = [(f, lambda ws: e3.gated_fwd(x, W, ws=ws)), (bw, lambda ws: e3.gated_bwd(x, W, dy, z, ws=ws)[1]),
             (rn, lambda ws: e3.residual_norm_bwd(None, dy, st, dy, pre=(b[:250].contiguous(), None), ws=ws)[4][0])]
    for nb, call in calls:
        assert nb > 0
        ref = call(None)
        assert torch.equal(call(torch.empty(nb, dtype=torch.uint8, device="cuda")), ref)
        with pytest.raises(e3.E3Error) as ei:
            call(torch.empty(nb - 1, dtype=torch.uint8, device="cuda"))
        assert ei.value.status == 4
        with pytest.raises(ValueError):
            call(torch.empty(nb, dtype=torch.uint8))
        with pytest.raises(TypeError):
            call(bytearray(nb))


def test_empty_rows_give_zero_sums(e3):  # noqa: F811
    import torch
    W = torch.randn(12, 20, device="cuda")
    none = torch.empty(0, 12, device="cuda")
    dy = torch.empty(0, 10, device="cuda")
    assert e3.gated_fwd(none, W).shape == (0, 10)
    dx, dW, db = e3.gated_bwd(none, W, dy, torch.empty(0, 20, device="cuda"))
    assert dx.shape == (0, 12) and not bool(dW.any()) and not bool(db.any()) and dW.shape == W.shape
    gate, w = torch.randn(10, device="cuda"), (torch.randn(10, device="cuda"), torch.randn(10, device="cuda"))
    s, y, st = e3.residual_norm_fwd(dy, dy, gate, 1.0, "layer", w, w, keep=("stats",))
    out = e3.residual_norm_bwd(dy, s, st, dy, dy, gate, 1.0, "layer", w, w)
    assert out[0].shape == (0, 10) and not bool(out[2].any())
    assert all(not bool(v.any()) for pair in out[3:] for v in pair)
    assert e3.dropout_fwd(dy, e3.Dropout(0.5, 1)).shape == (0, 10)
