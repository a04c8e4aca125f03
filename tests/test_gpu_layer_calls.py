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
