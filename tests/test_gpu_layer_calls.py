"""How the invariant layers' Python calls take their arguments."""
import pytest

from test_gpu_layers import e3  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def _inputs(m=300, k=32, n=24):
    import torch
    g = torch.Generator().manual_seed(1)
    return [torch.randn(s, generator=g).cuda() for s in ((m, k), (k, n), (m, n))]


def test_what_to_keep_may_be_any_iterable(e3):  # noqa: F811
    """A generator is gone after one look: what it names is kept all the same."""
    import torch
    x, W, dy = _inputs()
    for kind in (tuple, list, set, iter):
        y, z, z8 = e3.dense_fwd(x, W, act="silu", keep=kind(("z", "z8")))
        assert torch.equal(z, e3.dense_fwd(x, W)) and z8.shape == z.shape
        n, mean, rstd, x8 = e3.layer_norm_fwd(x, keep=kind(("stats", "x8")))
        assert x8.shape == x.shape
        dx, dW, db = e3.dense_bwd(x, W, dy, z, act="silu", want=kind(("dx", "db")))
        assert dW is None and dx.shape == x.shape and db.shape == (24,)
        dx, dg, db = e3.layer_norm_bwd(x8, None, x, mean, rstd, want=kind(("dgamma",)))
        assert dx is None and db is None and dg.shape == (32,)
    assert isinstance(e3.dense_fwd(x, W, keep=iter(())), torch.Tensor)
    with pytest.raises(ValueError):
        e3.dense_fwd(x, W, keep=iter(("x8",)))


def test_scratch_that_the_kernels_cannot_use_is_refused(e3):  # noqa: F811
    """Host memory, gaps in it, or no tensor at all: an error, before any launch.  Any element type will do;
    its size counts in bytes."""
    import torch
    x, W, dy = _inputs(3000, 300, 200)
    z = e3.dense_fwd(x, W)
    mean, rstd = e3.layer_norm_fwd(x, keep=("stats",))[1:]
    few, wide = x[:16].contiguous(), torch.randn(300, 500, device="cuda")
    few_long = torch.randn(16, 1000, device="cuda")
    W_long = torch.randn(1000, 500, device="cuda")
    nb = {"bwd": e3.dense_workspace_size(3000, 300, 200)[1], "fwd": e3.dense_workspace_size(16, 1000, 500)[0],
          "norm": e3.layer_norm_workspace_size(3000, 300)}
    assert min(nb.values()) > 0
    calls = {"bwd": lambda ws: e3.dense_bwd(x, W, dy, z, act="silu", ws=ws)[1],
             "fwd": lambda ws: e3.dense_fwd(few_long, W_long, ws=ws),
             "norm": lambda ws: e3.layer_norm_bwd(x, None, x, mean, rstd, ws=ws)[1]}
    for k, call in calls.items():
        for ws in (torch.empty(nb[k], dtype=torch.uint8), torch.empty(2 * nb[k], dtype=torch.uint8, device="cuda")[::2]):
            with pytest.raises(ValueError):
                call(ws)
        with pytest.raises(TypeError):
            call(bytearray(nb[k]))
        with pytest.raises(e3.E3Error) as ei:
            call(torch.empty(nb[k] - 1, dtype=torch.uint8, device="cuda"))
        assert ei.value.status == 4
        ref = call(None)
        for ws in (torch.empty(nb[k], dtype=torch.uint8, device="cuda"), torch.empty((nb[k] + 3) // 4, device="cuda")):
            assert torch.equal(call(ws), ref)
    # a call that needs none looks at what it is given all the same
    with pytest.raises(ValueError):
        e3.dense_fwd(few, wide, ws=torch.empty(16, dtype=torch.uint8))
