"""The loops of the invariant layers that only larger sizes take: outputs past the caches, several rounds
of a workgroup's rows."""
import pytest

from test_gpu_layers import e3  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


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
