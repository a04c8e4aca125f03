"""The float64 oracle of a residual block's layers: gradients against differences, the generator against its
authors' known answers, closed forms."""
import numpy as np
import pytest

from oracle import blocks as ob
from oracle import layers as ol


def _differences(f, args, cots, got, step=1e-5, bar=2e-7):
    """<cot, f> by central differences in a random direction of each argument against <got, direction>."""
    rng = np.random.default_rng(5)
    for i, g in got.items():
        d = rng.standard_normal(args[i].shape)
        ends = []
        for sign in (1, -1):
            a = list(args)
            a[i] = args[i] + sign * step * d
            ends.append(sum((c * o).sum() for c, o in zip(cots, f(*a))))
        num = (ends[0] - ends[1]) / (2 * step)
        assert abs(num - (g * d).sum()) < bar * max(1.0, abs(num)), i


@pytest.mark.parametrize("name", ol.ACTIVATIONS)
def test_gated_gradients_equal_differences(name):
    rng = np.random.default_rng(1)
    x, W, b, dy = (rng.standard_normal(s) for s in ((7, 5), (5, 12), (12,), (7, 6)))
    z = ob.gated_fwd(x, W, b, name)[1]
    dx, dW, db = ob.gated_bwd(x, W, dy, z, name)
    # relu's kink: no value of g within the step of it
    assert name != "relu" or np.abs(z[:, :6]).min() > 1e-3
    _differences(lambda x, W, b: (ob.gated_fwd(x, W, b, name)[0],), (x, W, b), (dy,), {0: dx, 1: dW, 2: db})


def test_gated_closed_form():
    y, z = ob.gated_fwd([[2.0, -1.0]], [[1, 0, 3, 0], [0, 1, 0, 5]], [0, 0, 1, 0], "relu")
    assert np.array_equal(z, [[2, -1, 7, -5]]) and np.array_equal(y, [[14, 0]])


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_generator_known_answers(counter, key, words):
    """The known-answer vectors that the generator's authors publish with it."""
    assert tuple(int(w) for w in ob.philox(counter, key)) == words


def test_mask_shares_and_keys():
    """The share of dropped values is p to five deviations; other seeds, offsets and rows have other masks; a
    column's bit does not depend on how many there are."""
    k = ob.kept(400, 1000, 0.3, 7, 5)
    assert abs((~k).mean() - 0.3) < 5 * np.sqrt(0.21 / k.size)
    for other in (ob.kept(400, 1000, 0.3, 8, 5), ob.kept(400, 1000, 0.3, 7, 6), ob.kept(400, 1000, 0.3, 7 + (1 << 32), 5),
                  ob.kept(np.arange(400) + (1 << 32), 1000, 0.3, 7, 5)):
        assert abs((k == other).mean() - 0.58) < 0.01
    assert np.array_equal(ob.kept(400, 37, 0.3, 7, 5), k[:, :37])
    assert ob.kept(5, 9, 0.0, 1).all() and not ob.kept(5, 9, 1.0, 1).any() and not ob.factors(5, 9, 1.0, 1).any()
    # neighbouring columns and rows are independent
    for a, b in ((k[:, 1:], k[:, :-1]), (k[1:], k[:-1]), (k[:, 8:], k[:, :-8])):
        assert abs((a & b).mean() - 0.49) < 0.01


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("post,pre", [(False, True), (True, False), (True, True), (False, False)])
@pytest.mark.parametrize("gate", ["none", "row", "full"])
@pytest.mark.parametrize("p", [0.0, 0.4])
def test_residual_norm_gradients_equal_differences(norm, post, pre, gate, p):
    rng = np.random.default_rng(2)
    M, K = 6, 9
    h, r, dy, ds = (rng.standard_normal((M, K)) for _ in range(4))
    g = rng.standard_normal(K if gate == "row" else (M, K))
    w = [1 + rng.standard_normal(K) for _ in range(4)]
    f = ob.factors(M, K, p, 11) if p else None

    def run(h, r, g, g1, b1, g2, b2):
        s, y, _, _ = ob.residual_norm_fwd(h, r, g if gate != "none" else None, 0.7, norm,
                                          (g1, b1 if norm == "layer" else None) if post else None,
                                          (g2, b2 if norm == "layer" else None) if pre else None, 1e-5, f)
        return (s, y) if pre else (s,)
    args = (h, r, g, *w)
    posts = (w[0], w[1] if norm == "layer" else None) if post else None
    pres = (w[2], w[3] if norm == "layer" else None) if pre else None
    s, y, first, last = ob.residual_norm_fwd(h, r, g if gate != "none" else None, 0.7, norm, posts, pres, 1e-5, f)
    d, dh, dgate, dpost, dpre = ob.residual_norm_bwd(h, s, first, last, dy if pre else None, ds,
                                                     g if gate != "none" else None, 0.7, norm, posts, pres, f)
    got = {0: dh, 1: d}
    if gate != "none":
        got[2] = dgate
    for k, v in ((3, dpost), (5, dpre)):
        if v is not None:
            got[k] = v[0]
            if norm == "layer":
                got[k + 1] = v[1]
    _differences(run, args, (ds, dy), got)


def test_residual_norm_closed_form():
    s, y, first, last = ob.residual_norm_fwd([[3.0, 4.0]], [[1.0, 1.0]], np.array([1.0, 2.0]), 0.5, "rms", (None, None),
                                             None, 0.0)
    assert np.allclose(first[1], [1 / np.sqrt(12.5)]) and y is None and last is None
    assert np.allclose(s, [[1 + 1.5 / np.sqrt(12.5), 1 + 4 / np.sqrt(12.5)]])
