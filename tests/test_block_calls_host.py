"""Host checks of how the gated layers, dropout and the residual norms are offered: their scratch and where their
names are found."""
import pytest

from paper_2609_35099_amd import e3mi


@pytest.mark.parametrize("dtype,M,K,N", [("bfloat16", 16384, 1024, 2048), ("float32", 100_000, 512, 512),
                                         ("float32", 200_000, 300, 400), ("bfloat16", 300_000, 200, 256)])
def test_gated_backward_scratch_holds_dz_once(dtype, M, K, N):
    """dz [M, 2 N]; beside it partial sums of db, 512 rows of it at most, and of the products: where their tiles are
    few their reductions are cut, into 256 tiles of 256 x 256 float32 or 512 of 128 x 128 at most (64 MB), with a
    row of column sums each."""
    dz = M * 2 * N * (4 if dtype == "float32" else 2)
    ws = e3mi.gated_workspace_size(M, K, N, dtype)[1]
    assert dz <= ws <= dz + (1 << 26) + 2 * 512 * 2 * N * 4 + 4096, (ws, dz)


def test_the_package_offers_the_layers():
    """Every call of the invariant layers, and what they take, is found in the package itself."""
    import paper_2609_35099_amd as package
    layers = [n for n in vars(e3mi) if n.startswith(("dense_", "layer_norm_", "gated_", "dropout_", "residual_norm_"))]
    assert {"gated_fwd", "gated_bwd", "gated_workspace_size", "dropout_fwd", "dropout_bwd", "residual_norm_fwd",
            "residual_norm_bwd", "residual_norm_workspace_size"} <= set(layers)
    for n in (*layers, "Dropout", "Packed8", "pack8", "unpack8"):
        assert n in package.__all__ and getattr(package, n) is getattr(e3mi, n), n
    assert all(hasattr(package, n) for n in package.__all__)
