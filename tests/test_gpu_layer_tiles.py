"""The tiles and row loops of the invariant layers that only larger sizes take, against float64.

Every case names the kernels that it is there for and checks, by the library's timings, that they ran:
a change of the rules that choose them fails here instead of leaving them untested.

The references are the operators' definitions in float64, by elementary operations on the device.  Bars
(relative L2 per output):
  float32   2e-6, as for the smaller sizes (sums of up to 100,000 terms go through tiles and splits).
  bfloat16  2e-3 and, for gradients, 3e-3 against the definition rounded as the calls say (outputs once,
            the dz of a gradient before its products): a few values cross a tie.
            Gradients against the definition with nothing rounded: rounding values of random mantissa to
            8 bits is an error of 2^-7 / sqrt(12) / 1.47 = 1.5e-3 of their size, 1.7e-3 at most over
            mantissas; dz and the output are rounded once each, independently: 2.4e-3 together, bar 3e-3.
"""
import numpy as np
import pytest

from oracle import layers as ol
from test_gpu_layers import TOL, TOL_BWD, dev, e3, near_steps, out_like  # noqa: F401 (e3: a fixture)

pytestmark = pytest.mark.gpu


def ran(e3, fn):
    """fn()'s result and the names of the kernels that it launched."""
    e3.timing_reset()
    e3.timing_enable(True)
    try:
        got = fn()
    finally:
        e3.timing_enable(False)
    names = set(e3.timing_read())
    e3.timing_reset()
    return got, names


def normal(*shape, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


def rows_of(t, dt, gap):
    """t in type dt as rows of a wider tensor (its other columns NaN), one element off its allocation."""
    import torch
    t = t.to(getattr(torch, dt))
    if not gap:
        return t
    m, n = t.shape
    buf = torch.full((m * (n + gap) + 1,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[1:].view(m, n + gap)[:, :n]
    v.copy_(t)
    return v


def rounded(v, dt):
    return v if dt == "float32" else v.bfloat16().double()


def values(e3, t):
    """A kept activation in float64."""
    import torch
    if not isinstance(t, e3.Packed8):
        return t.double()
    table = np.ldexp(1.0, np.arange(256) - 127)     # (a device's power function is not exact)
    table[255] = np.nan
    step = torch.from_numpy(table).cuda()[t.c.long()]
    return t.q.double() * step.repeat_interleave(32, 1)[:, : t.q.shape[1]]


def off(got, ref):
    """Relative L2 distance."""
    return float((got.double() - ref).norm() / ref.norm())


def silu(z):
    import torch
    s = torch.sigmoid(z)
    return z * s, s + z * s * (1 - s)


def gelu_slope(z):
    import torch
    return 0.5 * (1 + torch.erf(z / 2**0.5)) + z * torch.exp(-0.5 * z * z) / (2 * np.pi)**0.5


# ---------------------------------------------------------------- dense layers
# whole and ragged rows, columns and reductions; the last names say what is split along its reduction
FORWARD = [("bfloat16", 16383, 515, 1021, 6, {"dense_fwd_256"}), ("bfloat16", 16384, 256, 1024, 0, {"dense_fwd_256"}),
           ("bfloat16", 3001, 4099, 2051, 0, {"dense_fwd_256", "dense_join"}),
           ("bfloat16", 24001, 300, 515, 2, {"dense_fwd_128"}),
           ("bfloat16", 300, 9001, 300, 1, {"dense_fwd_128", "dense_join"}),
           ("float32", 40003, 130, 200, 3, {"dense_fwd_128"}), ("float32", 16384, 256, 1024, 0, {"dense_fwd_128"}),
           ("float32", 300, 4100, 300, 1, {"dense_fwd_128", "dense_join"})]


@pytest.mark.parametrize("dt,M,K,N,gap,names", FORWARD)
def test_dense_forward_tiles(e3, dt, M, K, N, gap, names):  # noqa: F811
    import torch
    x = normal(M, K, seed=1) * torch.exp(0.5 * normal(M, 1, seed=2)) + 0.2
    xd, Wd, bd = rows_of(x, dt, gap), dev(normal(K, N, seed=3).cpu() / K**0.5, dt), dev(0.3 * normal(N, seed=4).cpu(), dt)
    rd = rows_of(normal(M, N, seed=5), dt, gap)
    xd[5, K - 1], xd[M - 2, 0] = float("inf"), float("nan")    # a row in the middle of a tile, one in the last
    print("[case] dense_fwd tiles", dt, M, K, N, gap, flush=True)
    out, untouched = out_like((M, N), dt, gap, 1 if gap else 0)
    (_, z, z8, y8), got = ran(e3, lambda: e3.dense_fwd(xd, Wd, bd, rd, act="silu", keep=("z", "z8", "y8"), out=out))
    assert got == names
    ref = xd.double() @ Wd.double()
    fine = torch.isfinite(ref)
    assert int(fine.sum()) == (M - 2) * N and not bool(fine[5].any()) and not bool(fine[M - 2].any())
    zr = ref + bd.double()
    yr = silu(zr)[0] + rd.double()
    assert untouched()
    assert off(z[fine], rounded(zr[fine], dt)) < TOL[dt] and off(out[fine], rounded(yr[fine], dt)) < TOL[dt]
    assert bool(torch.isnan(out[M - 2]).all())
    at = torch.cat([torch.arange(6, 300), torch.randint(300, M - 2, (1000,)) if M > 300 else torch.arange(0), torch.tensor([M - 1])])
    at = at[(at != M - 2) & (at < M)].cuda()
    near_steps(e3.Packed8(z8.q[at], z8.c[at]), zr[at].cpu().numpy())
    q, c = ol.pack8(out[at].double().cpu().numpy())
    assert np.array_equal(y8.q[at].cpu().numpy(), q) and np.array_equal(y8.c[at].cpu().numpy(), c)
    # without the extra outputs, into fresh memory: the same bits
    assert torch.equal(torch.nan_to_num(e3.dense_fwd(xd, Wd, bd, rd, act="silu")), torch.nan_to_num(out))
    # the bare product; its infinities are the definition's
    y = e3.dense_fwd(xd, Wd)
    assert off(y[fine], rounded(ref[fine], dt)) < TOL[dt]
    assert torch.equal(y[5].double(), ref[5]) and bool(torch.isnan(y[M - 2]).all())


# dx and dW tiles; K up to 256: dz formed by the products' loads (bfloat16 from packed z: up to 128, or few
# columns); above: written once
BACKWARD = [("bfloat16", 12289, 1030, 2051, 0, {"dense_dz", "dense_bwd_dx_256", "dense_bwd_dw_256", "dense_join"}),
            ("bfloat16", 45057, 250, 2051, 2, {"dense_bwd_dx_128", "dense_bwd_dw_256", "column_sums"}),
            ("bfloat16", 50021, 250, 1021, 3, {"dense_bwd_dx_256", "dense_bwd_dw_128", "column_sums"}),
            ("bfloat16", 3001, 2051, 4099, 1, {"dense_dz", "dense_bwd_dx_256", "dense_bwd_dw_128", "dense_join"}),
            ("bfloat16", 24001, 300, 515, 2, {"dense_dz", "dense_bwd_dx_128", "dense_bwd_dw_128", "column_sums"}),
            ("bfloat16", 16384, 512, 1024, 0, {"dense_dz", "dense_bwd_dx_128", "dense_bwd_dw_128", "dense_join"}),
            ("bfloat16", 300, 300, 9001, 0, {"dense_dz", "dense_bwd_dx_128", "dense_bwd_dw_64", "dense_join"}),
            ("float32", 40003, 130, 200, 3, {"dense_bwd_dx_128", "dense_bwd_dw_128", "column_sums"}),
            ("float32", 40003, 300, 200, 1, {"dense_dz", "dense_bwd_dx_128", "dense_bwd_dw_128", "column_sums"}),
            ("float32", 65536, 128, 256, 0, {"dense_bwd_dx_128", "dense_bwd_dw_128", "column_sums"}),
            ("float32", 300, 300, 4100, 0, {"dense_dz", "dense_bwd_dx_128", "dense_bwd_dw_64", "dense_join"})]


@pytest.mark.parametrize("dt,M,K,N,gap,names", BACKWARD)
@pytest.mark.parametrize("ckpt", [False, True])
def test_dense_backward_tiles(e3, dt, M, K, N, gap, names, ckpt):  # noqa: F811
    import torch
    xd, Wd = rows_of(normal(M, K, seed=1) + 0.2, dt, gap), dev(normal(K, N, seed=2).cpu() / K**0.5, dt)
    dyd, zd = rows_of(1e-3 * normal(M, N, seed=3), dt, gap), rows_of(normal(M, N, seed=4), dt, gap)
    xin, zin = (e3.pack8(xd), e3.pack8(zd)) if ckpt else (xd, zd)
    xr, zr, Wr, dyr = values(e3, xin), values(e3, zin), Wd.double(), dyd.double()
    for act in ("none", "silu", "gelu"):
        print("[case] dense_bwd tiles", dt, M, K, N, gap, ckpt, act, flush=True)
        z = None if act == "none" else zin
        dx, untouched = out_like((M, K), dt, gap, 1 if gap else 0)
        got, launched = ran(e3, lambda: e3.dense_bwd(xin, Wd, dyd, z, act=act, dx=dx))
        if act != "none":
            # (the join of a split product or the sums of many splits run beside them, whichever a size takes)
            if dt == "bfloat16" and ckpt and K > 128:
                names = names | {"dense_dz"}
            assert names - {"dense_join", "column_sums"} == launched - {"dense_join", "column_sums"}, launched
            assert names <= launched
        assert untouched()
        dz = dyr if act == "none" else dyr * (silu(zr)[1] if act == "silu" else gelu_slope(zr))
        db = dz.sum(0)
        # a column's terms may cancel: against their size
        size = float(db.norm() + 0.1 * (dz * dz).sum(0).sqrt().norm())
        assert float((got[2].double() - rounded(db, dt)).norm()) <= TOL_BWD[dt] * size
        for dzr, end in ((rounded(dz, dt), lambda v: rounded(v, dt)), (dz, lambda v: v)):
            for g, w in ((got[0], dzr @ Wr.t().contiguous()), (got[1], xr.t().contiguous() @ dzr)):
                assert off(g, end(w)) < TOL_BWD[dt], act
        # each alone, where the others' kernels do not run: the same bits
        for k, w in enumerate(("dx", "dW", "db")):
            one = e3.dense_bwd(xin if w == "dW" else None, Wd, dyd, z, act=act, want=(w,))
            assert torch.equal(one[k], got[k]), (act, w)


@pytest.mark.parametrize("K,N,names", [(64, 320, {"dense_fwd_panel"}), (64, 832, {"dense_fwd_shared", "dense_fwd_panel"}),
                                       (40, 300, {"dense_fwd_panel"}), (40, 400, {"dense_fwd_shared", "dense_fwd_panel"}),
                                       (64, 512, {"dense_fwd_shared"}), (32, 384, {"dense_fwd_shared"}),
                                       (32, 320, {"dense_fwd_panel"})])
def test_columns_past_the_shared_ones(e3, K, N, names):  # noqa: F811
    """Row blocks shared by four waves, and a second launch for the columns past the last 256 where that pays."""
    import torch
    xd, Wd, bd = normal(100003, K, seed=1), normal(K, N, seed=2) / K**0.5, normal(N, seed=3)
    print("[case] dense_fwd, shared row blocks", K, N, flush=True)
    y, launched = ran(e3, lambda: e3.dense_fwd(xd, Wd, bd, act="silu"))
    assert launched == names
    assert off(y, silu(xd.double() @ Wd.double() + bd.double())[0]) < TOL["float32"]
    assert torch.equal(e3.dense_fwd(xd, Wd, bd, act="silu", keep=("z8",))[0], y)


@pytest.mark.parametrize("dt,M,K,N,ckpt,once", [("bfloat16", 50021, 250, 1021, True, True), ("bfloat16", 50021, 250, 1021, False, False),
                                                ("bfloat16", 8001, 200, 300, True, True), ("bfloat16", 3001, 200, 300, True, False), ("bfloat16", 60003, 160, 64, True, True),
                                                ("bfloat16", 45011, 192, 64, True, False), ("bfloat16", 50021, 128, 1021, True, False),
                                                ("float32", 50021, 250, 300, True, False), ("float32", 9001, 260, 300, False, True)])
def test_dz_is_written_where_forming_it_is_slow(e3, dt, M, K, N, ckpt, once):  # noqa: F811
    """Formed per tile from 8 bits, bfloat16 took up to five times as long past 128 columns of x; the
    gradients are right either way."""
    import torch
    xd, Wd = rows_of(normal(M, K, seed=1), dt, 0), dev(normal(K, N, seed=2).cpu() / K**0.5, dt)
    dyd, zd = rows_of(1e-3 * normal(M, N, seed=3), dt, 0), rows_of(normal(M, N, seed=4), dt, 0)
    zin = e3.pack8(zd) if ckpt else zd
    print("[case] dense_bwd, dz written or formed", dt, M, K, N, ckpt, flush=True)
    got, names = ran(e3, lambda: e3.dense_bwd(xd, Wd, dyd, zin, act="gelu"))
    assert ("dense_dz" in names) == once
    dz = dyd.double() * gelu_slope(values(e3, zin))
    dzr = rounded(dz, dt)
    for g, w in zip(got, (dzr @ Wd.double().t().contiguous(), xd.double().t().contiguous() @ dzr)):
        assert off(g, rounded(w, dt)) < TOL_BWD[dt]
    size = float(dz.sum(0).norm() + 0.1 * (dz * dz).sum(0).sqrt().norm())
    assert float((got[2].double() - rounded(dz.sum(0), dt)).norm()) <= TOL_BWD[dt] * size
    for k, w in enumerate(("dx", "dW", "db")):
        assert torch.equal(e3.dense_bwd(xd if w == "dW" else None, Wd, dyd, zin, act="gelu", want=(w,))[k], got[k]), w


@pytest.mark.parametrize("dt,M,K,N,name", [("float32", 140001, 8, 64, "dense_thin"), ("bfloat16", 270001, 16, 64, "dense_thin"),
                                           ("float32", 262149, 64, 64, "dense_fwd_panel"),
                                           ("bfloat16", 262149, 128, 64, "dense_fwd_panel"),
                                           ("float32", 70001, 32, 256, "dense_fwd_shared"),
                                           ("float32", 70001, 64, 832, "dense_fwd_shared"),
                                           ("bfloat16", 45057, 250, 2051, "dense_fwd_256"),
                                           ("float32", 40003, 130, 256, "dense_fwd_128")])
def test_outputs_beside_y_do_not_change_it(e3, dt, M, K, N, name):  # noqa: F811
    """y alone past the caches goes by loops of its own: the same bits as beside z, z8 and y8."""
    import torch
    xd, Wd, bd = rows_of(normal(M, K, seed=1), dt, 0), dev(normal(K, N, seed=2).cpu() / K**0.5, dt), dev(normal(N, seed=3).cpu(), dt)
    for act in ol.ACTIVATIONS:
        print("[case] dense_fwd, alone and beside", dt, M, K, N, act, flush=True)
        y, names = ran(e3, lambda: e3.dense_fwd(xd, Wd, bd, act=act))
        assert name in names
        assert torch.equal(e3.dense_fwd(xd, Wd, bd, act=act, keep=("z", "z8", "y8"))[0], y), act


@pytest.mark.parametrize("M,K,N", [(40003, 130, 200), (300, 4100, 300)])
def test_float32_tiles_fall_back_for_large_operands(e3, M, K, N):  # noqa: F811
    """Operands of 1e32 leave the range of the scaled terms: the sums come from float32 arithmetic."""
    xd, Wd, dyd = dev(normal(M, K, seed=1).cpu(), "float32"), dev(normal(K, N, seed=2).cpu(), "float32"), dev(normal(M, N, seed=3).cpu(), "float32")
    xd[17] *= 1e32
    dyd[M - 1] *= 1e32
    print("[case] dense float32, large rows", M, K, N, flush=True)
    y, (dx, dW, db) = e3.dense_fwd(xd, Wd), e3.dense_bwd(xd, Wd, dyd)
    yr, dxr = xd.double() @ Wd.double(), dyd.double() @ Wd.double().t().contiguous()
    for g, w in ((y[17], yr[17]), (dx[M - 1], dxr[M - 1]), (db, dyd.double().sum(0))):
        assert off(g / 1e32, w / 1e32) < 1e-5       # sums of up to 4,100 terms one by one
    assert off(y[18:], yr[18:]) < TOL["float32"] and off(dx[:-1], dxr[:-1]) < TOL["float32"]
    assert bool((dW.double() - xd.double().t().contiguous() @ dyd.double()).isfinite().all())


# ---------------------------------------------------------------- layer norm and checkpoints
# outputs past the caches (non-temporal stores) and rows for several rounds of the backward's 512 workgroups,
# at widths that fill the registers' pieces exactly ("layer_norm_bwd_stream": loads and stores without
# branches) and that do not, and rows past the registers
NORM = [("bfloat16", 20001, 1024, 0, "layer_norm_bwd_stream"), ("bfloat16", 300001, 64, 0, "layer_norm_bwd_stream"),
        ("bfloat16", 5001, 4096, 8, "layer_norm_bwd_stream"), ("bfloat16", 2003, 16384, 0, "layer_norm_bwd_wide"),
        ("bfloat16", 2503, 8192, 0, "layer_norm_bwd_stream"), ("bfloat16", 2003, 10001, 2, "layer_norm_bwd_wide"),
        ("bfloat16", 40001, 515, 3, "layer_norm_bwd"), ("bfloat16", 1100, 16390, 0, "layer_norm_bwd_wide"),
        ("float32", 70003, 128, 4, "layer_norm_bwd_stream"), ("float32", 9001, 1024, 0, "layer_norm_bwd_stream"),
        ("float32", 2501, 4096, 0, "layer_norm_bwd_stream"), ("float32", 2003, 8192, 0, "layer_norm_bwd_stream"),
        ("float32", 40001, 515, 0, "layer_norm_bwd"), ("float32", 9001, 1025, 1, "layer_norm_bwd"),
        ("float32", 600, 16385, 0, "layer_norm_bwd_wide")]


@pytest.mark.parametrize("dt,rows,cols,gap,name", NORM)
@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm_many_rows(e3, dt, rows, cols, gap, name, affine):  # noqa: F811
    import torch
    assert rows * cols * (4 if dt == "float32" else 2) > 32 << 20
    xd = rows_of(normal(rows, cols, seed=1) * torch.exp(normal(rows, 1, seed=2)) + 0.5, dt, gap)
    dyd = rows_of(1e-3 * normal(rows, cols, seed=3), dt, gap)
    gd, bd = ((1 + 0.3 * normal(cols, seed=4)).to(xd.dtype), normal(cols, seed=5).to(xd.dtype)) if affine else (None, None)
    g, b = (gd.double(), bd.double()) if affine else (torch.ones(cols, device="cuda").double(), 0.0)
    x, dy = xd.double(), dyd.double()
    print("[case] layer norm, many rows", dt, rows, cols, gap, affine, flush=True)
    out, untouched = out_like((rows, cols), dt, gap, 1 if gap else 0)
    _, mean, rstd, x8, y8 = e3.layer_norm_fwd(xd, gd, bd, 1e-5, keep=("stats", "x8", "y8"), out=out)
    mr = x.mean(1)
    d = x - mr[:, None]
    rr = 1 / torch.sqrt((d * d).mean(1) + 1e-5)
    assert untouched()
    assert off(out, rounded(d * rr[:, None] * g + b, dt)) < TOL[dt]
    assert off(mean, mr) < 1e-6 and off(rstd, rr) < 1e-6
    at = torch.cat([torch.arange(64), torch.randint(64, rows, (200,)), torch.arange(rows - 64, rows)]).cuda()
    for p, v in ((x8, xd), (y8, out)):
        q, c = ol.pack8(v[at].double().cpu().numpy())
        assert np.array_equal(p.q[at].cpu().numpy(), q) and np.array_equal(p.c[at].cpu().numpy(), c)
    assert torch.equal(e3.layer_norm_fwd(xd, gd, bd), out)
    for xin in (xd, x8):
        dx, untouched = out_like((rows, cols), dt, gap, 1 if gap else 0)
        got, launched = ran(e3, lambda: e3.layer_norm_bwd(xin, gd, dyd, mean, rstd, dx=dx))
        assert name in launched and untouched()
        n = (values(e3, xin) - mean.double()[:, None]) * rstd.double()[:, None]
        a = dy * g
        ref = rstd.double()[:, None] * (a - a.mean(1, keepdim=True) - n * (a * n).mean(1, keepdim=True))
        assert off(dx, rounded(ref, dt)) < TOL[dt]
        for v, terms in ((got[1], dy * n), (got[2], dy)):
            w = terms.sum(0)
            # the terms of a column may cancel: against their size
            bar = TOL[dt] * float(w.norm()) + 2e-7 * float((terms * terms).sum(0).sqrt().norm())
            assert float((v.double() - rounded(w, dt)).norm()) <= bar


@pytest.mark.parametrize("dt,rows,cols", [("bfloat16", 20001, 1024), ("bfloat16", 300001, 64), ("bfloat16", 5001, 4096),
                                          ("float32", 70003, 128), ("float32", 9001, 1024), ("float32", 2003, 8192),
                                          ("float32", 40001, 515), ("float32", 600, 16385)])
@pytest.mark.parametrize("affine", [True, False])
def test_layer_norm_single_gradients_keep_their_bits(e3, dt, rows, cols, affine):  # noqa: F811
    """A gradient asked for alone, or with any others, has the same bits: also where dx streams."""
    import torch
    xd = rows_of(normal(rows, cols, seed=1) + 0.5, dt, 0)
    dyd = rows_of(1e-3 * normal(rows, cols, seed=3), dt, 0)
    gd = (1 + 0.3 * normal(cols, seed=4)).to(xd.dtype) if affine else None
    print("[case] layer norm, single gradients", dt, rows, cols, affine, flush=True)
    _, mean, rstd, x8 = e3.layer_norm_fwd(xd, gd, None, 1e-5, keep=("stats", "x8"))
    names = ("dx", "dgamma", "dbeta")
    for xin in (xd, x8):
        full = e3.layer_norm_bwd(xin, gd, dyd, mean, rstd)
        for want in (("dx",), ("dgamma",), ("dbeta",), ("dgamma", "dbeta"), ("dx", "dbeta")):
            got = e3.layer_norm_bwd(xin, gd, dyd, mean, rstd, want=want)
            assert all(torch.equal(got[k], full[k]) for k in range(3) if names[k] in want), want


@pytest.mark.parametrize("dt,rows,cols", [("bfloat16", 40001, 515), ("float32", 20001, 515), ("bfloat16", 9001, 2048),
                                          ("float32", 9001, 1024)])
def test_checkpoints_past_the_caches(e3, dt, rows, cols):  # noqa: F811
    import torch
    x = rows_of(normal(rows, cols, seed=1) * torch.exp(4 * normal(rows, 1, seed=2)), dt, 0)
    print("[case] pack8, many rows", dt, rows, cols, flush=True)
    p = e3.pack8(x)
    q, c = ol.pack8(x.double().cpu().numpy())
    assert np.array_equal(p.q.cpu().numpy(), q) and np.array_equal(p.c.cpu().numpy(), c)
    out, untouched = out_like((rows, cols), dt, 5, 3)
    e3.unpack8(p, out=out)
    assert untouched() and torch.equal(out.double(), values(e3, p))
    assert torch.equal(e3.unpack8(p, out.dtype), out)


@pytest.mark.parametrize("cols", [7, 32, 64, 100, 256, 515, 700, 1025, 2049, 4100, 8192, 20000])
def test_layer_norm_of_a_large_mean(e3, cols):  # noqa: F811
    """A mean 3,000 times the deviation: as a float32 it is off by up to 1e-4 deviations, which may not reach
    y.  x less any float32 near its mean is exact, so what is left is the rounding of sums of deviations:
    the bar of other inputs."""
    import torch
    x = (normal(40, cols, seed=cols) + 3000 * torch.linspace(1, 2, 40, device="cuda")[:, None]).contiguous()
    print("[case] layer norm, large mean", cols, flush=True)
    y, mean, rstd = e3.layer_norm_fwd(x, keep=("stats",))
    d = x.double() - x.double().mean(1, keepdim=True)
    r = 1 / torch.sqrt((d * d).mean(1) + 1e-5)
    assert off(y, d * r[:, None]) < TOL["float32"]
    assert off(mean, x.double().mean(1)) < 6e-8 and off(rstd, r) < 1e-6      # the mean: one rounding


# W shorter than a load's 16 bytes (a layer of one or two columns to a few): few rows, many, ragged
@pytest.mark.parametrize("dt", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,K,N,gap", [(9, 1, 1, 0), (40, 1, 3, 2), (1003, 3, 1, 0), (20011, 1, 2, 1), (300001, 1, 3, 0), (270001, 3, 1, 5)])
@pytest.mark.parametrize("ckpt", [False, True])
def test_dense_backward_of_a_short_matrix(e3, dt, M, K, N, gap, ckpt):  # noqa: F811
    """The sums over many rows go through tiles and splits as those of wider layers do (a wave for each took
    5 ms for a million rows).  A bfloat16 value is off by half a step, 2^-8 of it, at most."""
    import torch
    bar = 2e-6 if dt == "float32" else 1.001 * 2**-8
    xd, Wd = rows_of(normal(M, K, seed=1) + 0.2, dt, gap), dev(normal(K, N, seed=2).cpu(), dt)
    dyd, zd = rows_of(1e-3 * normal(M, N, seed=3), dt, gap), rows_of(normal(M, N, seed=4), dt, gap)
    xin, zin = (e3.pack8(xd), e3.pack8(zd)) if ckpt else (xd, zd)
    xr, zr, Wr, dyr = values(e3, xin), values(e3, zin), Wd.double(), dyd.double()
    for act in ("none", "gelu"):
        print("[case] dense_bwd, short W", dt, M, K, N, gap, ckpt, act, flush=True)
        z = None if act == "none" else zin
        dx, untouched = out_like((M, K), dt, gap, 1 if gap else 0)
        got, names = ran(e3, lambda: e3.dense_bwd(xin, Wd, dyd, z, act=act, dx=dx))
        assert ("dense_bwd_tiny" in names) == (M < 5000) and untouched()
        dz = dyr if act == "none" else dyr * gelu_slope(zr)
        dzr = rounded(dz, dt)
        assert off(dx, rounded(dzr @ Wr.t().contiguous(), dt)) < TOL_BWD[dt]
        for g, w, terms in ((got[1], xr.t().contiguous() @ dzr, (xr**2).t().contiguous() @ dzr**2), (got[2], dz.sum(0), (dz**2).sum(0))):
            assert bool(((g.double() - w).abs() <= bar * (w.abs() + terms.sqrt())).all())
        for k, w in enumerate(("dx", "dW", "db")):
            one = e3.dense_bwd(xin if w == "dW" else None, Wd, dyd, z, act=act, want=(w,))
            assert torch.equal(one[k], got[k]), (act, w)
