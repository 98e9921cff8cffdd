"""CPU pins of the references that the gated delta rule and the norms around a block are tested against: closed forms and central
differences (step 1e-5 in 64 bits: truncation 1e-10, rounding 1e-11 of the loss, held to 1e-6 of the gradient)."""
import numpy as np
import pytest

from _delta_ref import delta_bwd, delta_fwd, norm_bwd, norm_fwd


def _inputs(rng, L, Hk, Hv, dk, dv):
    k = rng.normal(size=(L, Hk, dk))
    return [rng.normal(size=(L, Hk, dk)), k / np.linalg.norm(k, axis=-1, keepdims=True), rng.normal(size=(L, Hv, dv)),
            -rng.uniform(0, 1, (L, Hv)), rng.uniform(0, 1, (L, Hv))]


def test_orthonormal_keys_store_their_values():
    rng = np.random.default_rng(0)
    k = np.linalg.qr(rng.normal(size=(6, 6)))[0][:, None, :]
    v = rng.normal(size=(6, 1, 4))
    o, states, _ = delta_fwd(k, k, v, np.zeros((6, 1)), np.ones((6, 1)), 1.0)
    assert np.allclose(o, v, atol=1e-12)                          # a key that was just written reads its value
    assert np.allclose(np.einsum("tk,kv->tv", k[:, 0], states[-1][0]), v[:, 0], atol=1e-12)


def test_overwriting_a_key_and_forgetting():
    rng = np.random.default_rng(1)
    k, v = rng.normal(size=(1, 1, 5)), rng.normal(size=(2, 1, 3))
    k = np.repeat(k / np.linalg.norm(k), 2, 0)
    o, _, _ = delta_fwd(k, k, v, np.zeros((2, 1)), np.ones((2, 1)), 1.0)
    assert np.allclose(o[1], v[1], atol=1e-12)                    # beta = 1: the new value replaces the old one
    s0 = rng.normal(size=(1, 5, 3))
    with np.errstate(invalid="raise"):
        o, _, _ = delta_fwd(k[:1], k[:1], v[:1], np.full((1, 1), -np.inf), np.full((1, 1), 0.5), 1.0, s0)
    assert np.allclose(o[0], 0.5 * v[0], atol=1e-12)              # nothing of the first state is left


@pytest.mark.parametrize("Hk,Hv", [(2, 2), (1, 3)])
def test_delta_gradients_are_differences(Hk, Hv):
    rng = np.random.default_rng(2)
    L, dk, dv = 7, 4, 3
    args = _inputs(rng, L, Hk, Hv, dk, dv) + [rng.normal(size=(Hv, dk, dv))]
    do, dl = rng.normal(size=(L, Hv, dv)), rng.normal(size=(Hv, dk, dv))

    def loss(a):
        o, st, _ = delta_fwd(*a[:5], 0.7, a[5])
        return (o * do).sum() + (st[-1] * dl).sum()

    grads = delta_bwd(*args[:5], 0.7, do, args[5], dl)
    for i, name in enumerate(("dq", "dk", "dv", "dg", "dbeta", "ds0")):
        got = np.zeros_like(args[i])
        for at in np.ndindex(args[i].shape):
            ends = []
            for s in (1e-5, -1e-5):
                a = [x.copy() for x in args]
                a[i][at] += s
                ends.append(loss(a))
            got[at] = (ends[0] - ends[1]) / 2e-5
        assert np.abs(got - grads[name]).max() <= 1e-6 * np.abs(grads[name]).max(), name


@pytest.mark.parametrize("post,groups,act", [("full", 1, "silu"), ("shared", 2, "sigmoid"), ("full", 3, "silu")])
def test_norm_gradients_are_differences(post, groups, act):
    rng = np.random.default_rng(3)
    M, D = 3, 6
    kw = dict(post=rng.normal(size=D // groups if post == "shared" else D), gate=rng.normal(size=(M, D)),
              residual=rng.normal(size=(M, D)), scale=rng.normal(size=D), pre=rng.normal(size=D))
    x, dh, dy = (rng.normal(size=(M, D)) for _ in range(3))

    def loss(x, kw):
        h, y, _ = norm_fwd(x, groups=groups, act=act, **kw)
        return (h * dh).sum() + (y * dy).sum()

    grads = norm_bwd(dh, dy, x, groups=groups, act=act, **kw)
    names = dict(x="dx", post="dpost_weight", gate="dgate", residual="dresidual", scale="dres_scale", pre="dpre_weight")
    for n, gn in names.items():
        base = x if n == "x" else kw[n]
        got = np.zeros_like(base)
        for at in np.ndindex(base.shape):
            ends = []
            for s in (1e-5, -1e-5):
                c = base.copy()
                c[at] += s
                ends.append(loss(c, kw) if n == "x" else loss(x, dict(kw, **{n: c})))
            got[at] = (ends[0] - ends[1]) / 2e-5
        assert np.abs(got - grads[gn]).max() <= 1e-6 * np.abs(grads[gn]).max(), n
