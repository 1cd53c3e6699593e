"""The float64 forms of the norms, the 8-bit set and the router (oracle/training_oracle.py): gradients against central differences,
the 8-bit form against its stated bounds."""
import numpy as np
import pytest

from oracle import training_oracle as R


def differences(f, x, step=1e-5):
    """Central differences of a scalar function, entry by entry."""
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradients_are_differences(rms):
    rng = np.random.default_rng(5)
    h, gain, bias, dy, dres = rng.normal(1.0, 2.0, (3, 7)), rng.normal(size=7), rng.normal(size=7), rng.normal(size=(3, 7)), rng.normal(size=(3, 7))
    loss = lambda h, gain, bias: float((R.norm_forward(h, gain, bias, 1e-5, rms)[0] * dy).sum() + (h * dres).sum())
    dh, dgain, dbias = R.norm_backward(h, gain, 1e-5, dy, dres, rms)
    # (differences of step 1e-5: truncation ~1e-10, rounding ~1e-15 / 1e-5 = 1e-10, both on values of size 10)
    assert np.allclose(dh, differences(lambda v: loss(v, gain, bias), h), atol=1e-7)
    assert np.allclose(dgain, differences(lambda v: loss(h, v, bias), gain), atol=1e-7)
    assert np.allclose(dbias, differences(lambda v: loss(h, gain, v), bias), atol=1e-7)


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("k", [1, 3, 5])
def test_router_gradient_is_a_difference(renorm, k):
    rng = np.random.default_rng(k)
    logits, dw = rng.normal(size=(6, 5)), rng.normal(size=(6, k))
    logits[2, 1:4] = -np.inf                    # fewer experts than slots
    valid = np.array([1, 1, 1, 0, 1, 1])
    r = R.route(logits, k, valid, renorm)
    got = R.route_backward(r, dw, 1.7, renorm)

    def loss(v):                                # the choice, and with it coef, stays
        s = R.route(v, k, valid, renorm)
        assert np.array_equal(s["ids"], r["ids"])
        return float((s["weights"] * dw).sum() + 1.7 * (r["coef"] * s["p"].sum(axis=0)).sum())
    finite = np.where(np.isinf(logits), 0.0, logits)
    want = differences(lambda v: loss(np.where(np.isinf(logits), -np.inf, v)), finite)
    assert np.allclose(got, np.where(np.isinf(logits), 0.0, want), atol=1e-8)
    assert not got[3].any()


def test_router_of_nothing():
    r = R.route(np.full((3, 4), -np.inf), 2)
    assert r["loss"] == 0 and not r["counts"].any() and (r["order"] == -1).all() and (r["ids"] == -1).all()
    assert np.isclose(R.route(np.zeros((8, 4)), 4)["loss"], 1.0)               # all experts alike: 1


def test_8_bit_form():
    rng = np.random.default_rng(1)
    v = (rng.normal(size=(4, 70)) * 10.0 ** rng.integers(-6, 6, (4, 70))).astype(np.float32)
    v[0, :32] = 0
    v[1, 40] = np.inf
    v[2, 69] = np.nan
    v[3, 5] = np.float32(127.75)                # alone in its power of two: rounds to 128, held to 127
    v[3, :5] = v[3, 6:32] = 1
    q, e = R.pack8(v)
    back = R.unpack8(q, e)
    assert not back[0, :32].any() and np.isnan(back[1, 32:64]).all() and np.isnan(back[2, 64:]).all()
    assert q[3, 5] == 127 and back[3, 5] == 127.0
    fine = np.isfinite(back)
    step = np.repeat(2.0 ** (e.astype(np.float64) - 133), 32, axis=1)[:, :70]
    assert (np.abs(back - v)[fine] <= (np.where(np.abs(q) == 127, 1.0, 0.5) * step)[fine]).all()
    q2, e2 = R.pack8(back.astype(np.float32))
    assert np.array_equal(q2, q) and np.array_equal(e2, e)                      # saving again changes nothing


def test_mask_words():
    idx = np.array([[0, 31, 32, 69], [1, 2, 3, 4]])
    assert R.unpack_mask(R.pack_mask(idx, 70), 70) == idx.tolist()
