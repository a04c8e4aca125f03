"""How the gated layers, dropout and the residual norms are called: outputs in the memory of inputs, and the kernels
that sizes and alignments choose."""
import re

import pytest

from oracle import blocks as ob
from test_gpu_blocks import DTS, _host_pair, _pair, _residual_inputs, close, names_of
from test_gpu_layers import dev, e3, host  # noqa: F401 (e3: a fixture)

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- outputs in the memory of inputs
# (float32 rows stay in registers up to 6,144 columns, bfloat16 rows up to 8,192)
@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("cols", [24, 64, 515, 6144, 6147, 20000])
@pytest.mark.parametrize("norm,after,before,gate", [("rms", True, True, "row"), ("layer", True, True, "full"),
                                                   ("layer", True, False, "row"), ("rms", False, True, "row")])
def test_residual_norm_backward_in_place(e3, dt, cols, norm, after, before, gate):  # noqa: F811
    """Gradients written where a cotangent, h or s was are those written apart, and so are the sums over rows."""
    import torch
    h, r, g, post, pre, ds, dy = _residual_inputs(33, cols, norm, after, before, gate, True)
    hd, rd, gd, dsd, dyd = (dev(v, dt) for v in (h, r, g, ds, dy))
    post, pre = _pair(post, dt, 0), _pair(pre, dt, 0)
    drop, f = e3.Dropout(0.2, 3), ob.factors(33, cols, 0.2, 3)
    out = e3.residual_norm_fwd(hd, rd, gd, 0.5, norm, post, pre, 1e-5, drop, keep=("stats",))
    s, st = out[0], out[-1]

    def run(dres=None, dh=None, **at):
        a = {k: v if k not in at else at[k] for k, v in (("h", hd), ("s", s), ("dy", dyd if before else None), ("ds", dsd))}
        got = e3.residual_norm_bwd(a["h"], a["s"], st, a["dy"], a["ds"], gd, 0.5, norm, post, pre, drop, dres=dres, dh=dh)
        return [v for o in got for v in (o if isinstance(o, tuple) else (o,)) if v is not None]
    want = run()
    count, stats = 1 + (norm == "layer"), list(host(st))
    firsts = tuple(stats[:count]) if after else None
    lasts = tuple(stats[-count:]) if before else None
    firsts, lasts = (v if v is None or count == 2 else (None, v[0]) for v in (firsts, lasts))
    ref = ob.residual_norm_bwd(host(hd), host(s), firsts, lasts, host(dyd) if before else None, host(dsd), host(gd), 0.5,
                               norm, _host_pair(post), _host_pair(pre), f)
    there = [True, True, True, *(v is not None for w in (post, pre) if w for v in w)]
    ref = [v for o in ref if o is not None for v in (o if isinstance(o, tuple) else (o,))]
    ref = [v for v, t in zip(ref, there, strict=True) if t]
    assert len(ref) == len(want)
    for got, v in zip(want, ref):
        close(got, v, dt)
    places = {"ds": dsd, "h": hd, **({"dy": dyd, "s": s} if before else {})}
    for a in places:
        for b in places:
            print("[case] in place", dt, cols, norm, after, before, gate, a, b, flush=True)
            here = {k: v.clone() for k, v in places.items()}
            pairs = [(here[a], None), (None, here[a])] if a == b else [(here[a], here[b])]
            for dres, dh in pairs:
                for k, v in places.items():
                    here[k].copy_(v)
                got = run(dres, dh, **here)
                assert len(got) == len(want)
                for u, v in zip(got, want):
                    assert torch.equal(u, v), (a, b)


# ---------------------------------------------------------------- which kernels run
def launched(f):
    """The names of the kernels that f launches, mangled where a type's name is unknown to the profiler (bfloat16)."""
    import torch
    from torch.profiler import ProfilerActivity, profile
    f()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        f()
        torch.cuda.synchronize()
    names = {e.name for e in p.events() if e.device_type == torch.autograd.DeviceType.CUDA}
    assert names
    return names


def direct(f):
    """Whether f's dense products read their operands straight to LDS."""
    names = launched(f)
    some = {"k_dense_direct" in n for n in names if "k_dense" in n and "join" not in n and "k_dense_dz" not in n}
    assert len(some) == 1, names
    return some.pop()


def bf16(seed, *shape, gap=0):
    """Normal values; gap: elements between a row's end and the next one's start."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.randn(*shape, generator=g, device="cuda").bfloat16()
    if not gap:
        return v
    wide = torch.zeros(shape[0], shape[1] + gap, dtype=v.dtype, device="cuda")
    wide[:, :shape[1]] = v
    return wide[:, :shape[1]]


@pytest.mark.parametrize("M,N,red,want", [(16384, 1024, 512, False), (65536, 512, 512, False), (65536, 512, 1024, False),
                                          (16384, 2048, 1536, True), (65536, 512, 2048, True)])
def test_dx_goes_direct_from_long_reductions_only(e3, M, N, red, want):  # noqa: F811
    """(Short ones are up to a fifth faster the other way.)  M x N values of dx from `red` columns of dy."""
    W, dy = bf16(1, N, red), bf16(2, M, red)
    assert direct(lambda: e3.dense_bwd(None, W, dy, want=("dx",))) == want
    assert not direct(lambda: e3.dense_bwd(None, W, bf16(2, M, red, gap=1), want=("dx",)))


@pytest.mark.parametrize("K,N,M,want", [(4096, 4096, 512, False), (4096, 4096, 1024, False), (2048, 8192, 1024, False),
                                        (4096, 4096, 2048, True), (1024, 4096, 16384, True)])
def test_dw_goes_direct_from_many_rows_only(e3, K, N, M, want):  # noqa: F811
    x, W, dy = bf16(1, M, K), bf16(2, K, N), bf16(3, M, N)
    assert direct(lambda: e3.dense_bwd(x, W, dy, want=("dW",))) == want
    assert not direct(lambda: e3.dense_bwd(bf16(1, M, K, gap=1), W, dy, want=("dW",)))


def sums_columns(names):
    """Whether one of the products sums the columns of its second operand (the last argument of its Job)."""
    return any(re.search(r"3JobI\w*?ELb1EE|Job<[^<>]*, true>", n) for n in names)


@pytest.mark.parametrize("dt", DTS)
@pytest.mark.parametrize("M,K,N,gap", [(3000, 128, 150, 0), (700, 40, 200, 3), (20011, 256, 96, 0), (65536, 256, 1024, 0)])
def test_products_from_a_finished_dz_sum_nothing(e3, dt, M, K, N, gap):  # noqa: F811
    """The gated backward has summed db when its products run, and a plain layer's without db has nothing to sum: dW
    does not form column sums for nobody, and has the bits it has beside them."""
    import torch
    x, W, dy, z = (v.to(getattr(torch, dt)) for v in (bf16(1, M, K, gap=gap), bf16(2, K, 2 * N) / K ** 0.5,
                                                      bf16(3, M, N, gap=gap), bf16(4, M, 2 * N)))
    names = launched(lambda: e3.gated_bwd(x, W, dy, z))
    assert any("k_gated_dz" in n for n in names) and not sums_columns(names), names
    if M == 65536 and dt == "bfloat16":
        assert sum("k_dense_direct" in n for n in names) == 2, names          # dx and dW
    dx, dW, db = e3.gated_bwd(x, W, dy, z)
    pick = torch.tensor([0, 1, M // 2, M - 1]).cuda()
    dz = ob.gated_dz(host(dy), host(z))
    dzr = host(torch.from_numpy(dz).to(getattr(torch, dt))) if dt == "bfloat16" else dz
    close(dx[pick], dzr[pick.cpu().numpy()] @ host(W).T, dt)
    cols = slice(0, 2 * N, max(1, N // 8))
    close(dW[:, cols], host(x).T @ dzr[:, cols], dt)
    close(db, dz.sum(0), dt)

    d = z                              # any cotangent of a plain layer [K, 2 N]
    assert sums_columns(launched(lambda: e3.dense_bwd(x, W, d)))
    assert not sums_columns(launched(lambda: e3.dense_bwd(x, W, d, want=("dx", "dW"))))
    for a, b in zip(e3.dense_bwd(x, W, d)[:2], e3.dense_bwd(x, W, d, want=("dx", "dW"))[:2]):
        assert torch.equal(a, b)


@pytest.mark.parametrize("M,K,N", [(16384, 1600, 2048), (16384, 2048, 2056)])
def test_dense_products_straight_to_lds_have_the_same_bits(e3, M, K, N):  # noqa: F811
    """Whole aligned rows take the direct tiles and rows at odd strides the register ones, to the same sums."""
    import torch
    x, W, dy, b = bf16(1, M, K), bf16(2, K, N) / K ** 0.5, bf16(3, M, N), bf16(4, N)
    xo, dyo = bf16(1, M, K, gap=1), bf16(3, M, N, gap=1)
    calls = [(lambda x, dy: e3.dense_fwd(x, W, b, act="gelu"), True), (lambda x, dy: e3.dense_bwd(x, W, dy, want=("dW",))[1], True),
             (lambda x, dy: e3.dense_bwd(None, W, dy, want=("dx",))[0], N % 64 == 0)]
    for call, want in calls:
        print("[case] dense direct", M, K, N, want, flush=True)
        assert direct(lambda: call(x, dy)) == want and not direct(lambda: call(xo, dyo))
        assert torch.equal(call(x, dy), call(xo, dyo))
    rows, cols = torch.tensor([0, 255, 256, M - 1]).cuda(), slice(0, N, N // 7)
    close(calls[1][0](x, dy)[:, cols], host(x).T @ host(dy[:, cols]), "bfloat16")
    close(calls[2][0](x, dy)[rows], host(dy[rows]) @ host(W).T, "bfloat16")


# what is launched for whole aligned rows, for rows at odd strides, and whether the former's product is direct
@pytest.mark.parametrize("M,K,N,one,two", [
    (16387, 576, 1000, {"gated_fwd_direct"}, {"gated_fwd_256"}), (8200, 1088, 2056, {"gated_fwd_direct"}, {"gated_fwd_256"}),
    (2048, 4096, 2048, {"gated_fwd_split_256", "gated_fwd_join"}, {"gated_fwd_split_256", "gated_fwd_join"}),
    (2000, 4160, 2040, {"gated_fwd_split_256", "gated_fwd_join"}, {"gated_fwd_split_256", "gated_fwd_join"})])
def test_gated_products_straight_to_lds_have_the_same_bits(e3, M, K, N, one, two):  # noqa: F811
    import torch
    x, xo, W, b = bf16(1, M, K), bf16(1, M, K, gap=1), bf16(2, K, 2 * N) / K ** 0.5, bf16(3, 2 * N)
    print("[case] gated direct", M, K, N, flush=True)
    assert names_of(e3, lambda: e3.gated_fwd(x, W, b)) == one and names_of(e3, lambda: e3.gated_fwd(xo, W, b)) == two
    for v, fast in ((x, True), (xo, False)):
        names = launched(lambda: e3.gated_fwd(v, W, b))
        assert any("k_gated_direct" in n or "k_dense_direct" in n for n in names) == fast, names
    got, other = (e3.gated_fwd(v, W, b, keep=("z", "z8", "y8")) for v in (x, xo))
    for u, v in zip(got, other):
        for p, q in zip(u if isinstance(u, tuple) else (u,), v if isinstance(v, tuple) else (v,)):
            for r, s in ((p.q, q.q), (p.c, q.c)) if isinstance(p, e3.Packed8) else ((p, q),):
                assert torch.equal(r, s)
    assert torch.equal(e3.gated_fwd(x, W, b), got[0])
    rows = torch.tensor([0, 255, 256, M - 1]).cuda()
    y, z = ob.gated_fwd(host(x[rows]), host(W), host(b))
    close(got[0][rows], y, "bfloat16")
    close(got[1][rows], z, "bfloat16")
