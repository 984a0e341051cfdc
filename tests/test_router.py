"""Host-side checks of the router's entry points (include/routepack/router.h)
that need no GPU, and pins of their oracle: argument errors come before any
device work, and the oracle's formulas agree with small worked examples."""
import ctypes as C
import os
import re

import numpy as np
import pytest

from oracle import router as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOME = C.c_void_p(64)  # never read: every call below is refused, or has no work


def test_every_declared_entry_point_is_exported():
    import paper_2608_12146_amd as rp
    src = open(os.path.join(ROOT, "include", "routepack", "router.h")).read()
    names = re.findall(r"^(?:int|int64_t)\s+(routepack_\w+)\s*\(", src, re.M)
    assert sorted(names) == sorted(rp.ROUTER_EXPORTS)
    lib = rp.load_library()
    assert all(hasattr(lib, n) for n in names)


def _problem(N=2, L=3, E=16, k=2):
    import paper_2608_12146_amd as rp
    return rp.Problem(N, L, E, k, 1, 1, 1, [0], 64, [1], [0])


def _rows(type_, T=4, data=64, ts=48, ls=16):
    import paper_2608_12146_amd as rp
    return rp._Rows(data, type_, T, ts, ls)


def _route(prob, z, rec=None, bias=None, score=0, scale=1.0, ids=SOME, gates=SOME):
    import paper_2608_12146_amd as rp
    return rp.load_library().routepack_route_tokens(prob and prob.ref, z and C.byref(z), rec and C.byref(rec), bias,
                                                    score, 1, scale, ids, gates, None)


def test_route_refusals():
    F, I = _rows(0), _rows(5)
    assert _route(None, F) == -1 and _route(_problem(), None) == -1
    for bad in (_rows(3), _rows(-1), _rows(0, T=-1), _rows(0, data=None), _rows(0, ts=-1), _rows(0, ls=-4)):
        assert _route(_problem(), bad) == -1
    for bad in (_rows(0), _rows(7), _rows(5, T=3), _rows(5, data=None), _rows(5, ts=-2)):
        assert _route(_problem(), F, bad) == -1
    assert _route(_problem(), F, score=2) == -1 and _route(_problem(), F, scale=float("inf")) == -1
    assert _route(_problem(), F, I, bias=SOME) == -1
    assert _route(_problem(), F, ids=None) == -1 and _route(_problem(), F, gates=None) == -1
    for k in (0, -1, 17):
        assert _route(_problem(k=k), F) == -1
    assert _route(_problem(L=-1), F) == -1 and _route(_problem(E=0), F) == -1
    assert _route(_problem(E=2049), F) == -8 and _route(_problem(E=64, k=33), F) == -8
    # nothing to do: no pointer is needed
    assert _route(_problem(), _rows(0, T=0, data=None), ids=None, gates=None) == 0
    assert _route(_problem(L=0), _rows(0, data=None), ids=None, gates=None) == 0


def test_count_refusals():
    import paper_2608_12146_amd as rp
    f = rp.load_library().routepack_count_demand

    def call(prob, rec, off=SOME, out=SOME):
        return f(prob and prob.ref, rec and C.byref(rec), off, out, None)
    I = _rows(5)
    assert call(None, I) == -1 and call(_problem(), None) == -1
    for bad in (_rows(0), _rows(9), _rows(5, T=-1), _rows(5, data=None), _rows(5, ls=-1)):
        assert call(_problem(), bad) == -1
    assert call(_problem(), I, off=None) == -1 and call(_problem(), I, out=None) == -1
    assert call(_problem(k=0), I) == -1 and call(_problem(E=0), I) == -1
    assert call(_problem(N=-1), I) == -1 and call(_problem(L=-1), I) == -1
    assert call(_problem(E=16385), I) == -8 and call(_problem(), _rows(5, T=1 << 30)) == -8
    assert call(_problem(k=257), I) == -8
    assert call(_problem(N=0), I, None, None) == 0 and call(_problem(L=0), I, None, None) == 0


def test_balance_refusals():
    import paper_2608_12146_amd as rp
    lib = rp.load_library()

    def call(prob, z, G=2, off=SOME, counts=SOME, ctype=5, score=0, loss=SOME, shares=SOME, work=SOME, size=1 << 40):
        return lib.routepack_balance_loss(prob and prob.ref, z and C.byref(z), G, off, counts, ctype, score, loss,
                                          shares, work, size, None)
    F = _rows(0)
    assert call(None, F) == -1 and call(_problem(), None) == -1
    for more in (dict(G=0), dict(off=None), dict(counts=None), dict(ctype=4), dict(score=-1), dict(loss=None),
                 dict(shares=None), dict(work=None), dict(work=C.c_void_p(72)), dict(size=8)):
        assert call(_problem(), F, **more) == -1, more
    assert call(_problem(E=2049), F) == -8
    need = lib.routepack_balance_workspace(_problem().ref, 4, 2)
    assert need > 0 and call(_problem(), F, size=need - 1) == -1
    assert lib.routepack_balance_workspace(None, 4, 2) == -1
    assert lib.routepack_balance_workspace(_problem().ref, -1, 2) == -1
    assert lib.routepack_balance_workspace(_problem().ref, 4, 0) == -1
    assert call(_problem(L=0), F, loss=None) == 0


def test_backward_refusals():
    import paper_2608_12146_amd as rp
    lib = rp.load_library()

    def call(prob, z, rec=None, dg=None, scale=1.0, G=0, off=None, counts=None, ctype=0, dloss=None, score=0, out=SOME):
        return lib.routepack_route_backward(prob and prob.ref, z and C.byref(z), rec and C.byref(rec), dg, 1, scale, G,
                                            off, counts, ctype, dloss, score, out, None)
    F, I = _rows(0), _rows(5)
    loss = dict(G=2, off=SOME, counts=SOME, ctype=5, dloss=SOME)
    assert call(None, F, I, SOME) == -1 and call(_problem(), F) == -1
    assert call(_problem(), F, I) == -1 and call(_problem(), F, I, SOME, out=None) == -1
    assert call(_problem(), F, I, SOME, scale=float("nan")) == -1 and call(_problem(), F, I, SOME, score=3) == -1
    assert call(_problem(k=17), F, I, SOME) == -1 and call(_problem(E=64, k=40), F, I, SOME) == -8
    assert call(_problem(), F, _rows(5, T=5), SOME) == -1
    for more in (dict(G=0), dict(off=None), dict(counts=None), dict(ctype=3)):
        assert call(_problem(), F, **dict(loss, **more)) == -1
    assert call(_problem(), _rows(0, T=0, data=None), _rows(5, T=0, data=None), None, out=None) == 0


# -- pins of the oracle -------------------------------------------------------

def test_oracle_choices():
    z = np.array([[[1.0, 3.0, 3.0, -np.inf, np.nan]]])
    assert O.choose(z, 5).tolist() == [[[1, 2, 0, -1, -1]]]
    assert O.choose(z, 2, np.array([[5.0, 0.0, 0.1, 9.0, 9.0]]), "sigmoid").tolist() == [[[0, 2]]]
    assert O.choose(z, 3, np.array([[-np.inf, 0.0, np.nan, 9.0, 9.0]]), "softmax")[0, 0, 0] in (1, -1)


def test_oracle_gates():
    z = np.log(np.array([[[1.0, 2.0, 5.0]]]))
    ids = np.array([[[2, 0]]])
    assert np.allclose(O.gates(z, ids, "softmax", False, 2.0), [[[2 * 5 / 8, 2 / 8]]])
    assert np.allclose(O.gates(z, ids, "softmax", True, 1.0), [[[5 / 6, 1 / 6]]])
    s = np.array([5 / 6, 1 / 2])
    assert np.allclose(O.gates(z, ids, "sigmoid", False, 1.0), [[s]])
    assert np.allclose(O.gates(z, ids, "sigmoid", True, 1.0), [[s / s.sum()]])
    assert O.gates(z, np.array([[[-1, 3]]]), "sigmoid", True, 1.0).tolist() == [[[0.0, 0.0]]]


def test_oracle_balance():
    """Even scores and even counts give a loss of 1; all choices on one expert
    that has the whole score give E."""
    z = np.zeros((4, 1, 8))
    off = np.array([0, 1, 1, 4])
    loss, shares = O.balance(z, np.full((3, 1, 8), 7), off, "softmax")
    assert np.allclose(shares[[0, 2]], 1 / 8) and not shares[1].any() and np.allclose(loss, 2 / 3)
    z = np.full((4, 1, 8), -np.inf)
    z[:, :, 5] = 0.0
    counts = np.zeros((1, 1, 8))
    counts[0, 0, 5] = 32
    assert np.allclose(O.balance(z, counts, np.array([0, 4]), "softmax")[0], 8.0)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalize", [True, False])
def test_oracle_gradient(score, normalize):
    """The oracle's gradient against central differences (error of order h^2
    and 2^-53 / h), and within its own magnitude."""
    rng = np.random.default_rng(3)
    T, L, E, k, h = 5, 2, 7, 3, 1e-5
    z, dg = rng.normal(size=(T, L, E)), rng.normal(size=(T, L, k))
    ids = rng.integers(-1, E, size=(T, L, k))
    counts, off, dl = rng.integers(0, 9, size=(2, L, E)), np.array([0, 2, 4]), rng.random(L)

    def value(x):
        return (O.gates(x, ids, score, normalize, 1.5) * dg).sum() + (O.balance(x, counts, off, score)[0] * dl).sum()
    got, mag = O.backward(z, score, ids, dg, normalize, 1.5, counts, off, dl)
    for at in np.ndindex(*z.shape):
        up, down = z.copy(), z.copy()
        up[at] += h
        down[at] -= h
        assert abs((value(up) - value(down)) / (2 * h) - got[at]) < 1e-8
    assert (np.abs(got) <= mag * (1 + 1e-12) + 1e-300).all()


def test_oracle_counts():
    ids = np.array([[[0, 1]], [[1, 1]], [[-1, 9]], [[2, 0]]])
    assert O.count(ids, np.array([0, 2, 2, 3]), 3).tolist() == [[[1, 3, 0]], [[0, 0, 0]], [[0, 0, 0]]]


def test_oracle_biased_choices_over_nan_and_infinities():
    """Under a softmax a NaN logit takes no part in the scores that a bias is
    added to, and experts of +inf share them alone."""
    z = np.array([[[1.0, 3.0, 3.0, -np.inf, np.nan]], [[1.0, np.inf, 0.0, np.inf, np.nan]]])
    none = np.zeros((1, 5))
    with np.errstate(invalid="ignore"):
        ids = O.choose(z, 5, none, "softmax")
        assert ids.tolist() == [[[1, 2, 0, -1, -1]], [[1, 3, 0, 2, -1]]]
        some = np.array([[0.6, 0.0, 0.4, 0.0, 9.0]])
        assert O.choose(z[1:], 3, some, "softmax").tolist() == [[[0, 1, 3]]]
        assert O.choose(z[:1], 2, np.array([[-np.inf, 0.0, np.nan, 9.0, 9.0]]), "softmax").tolist() == [[[1, -1]]]
        # the gates: NaN where such a score enters
        g = O.gates(z, ids, "softmax", True, 1.0)
        assert np.isfinite(g[0]).all() and np.isnan(g[1, 0, :4]).all()
        g = O.gates(z, ids, "softmax", False, 1.0)
        assert np.isnan(g[0, 0, :3]).all() and np.isnan(g[1, 0, :4]).all() and not g[:, 0, 4].any()


def test_sizes_past_64_bits_are_refused():
    """Numbers of tokens, layers and groups whose products leave 64 bits (of
    broadcast logits, say) give an error, no size that wrapped around."""
    import paper_2608_12146_amd as rp
    lib = rp.load_library()
    most = 2 ** 31 - 1
    for T, L, E, G in ((4, 1 << 20, 2048, most), (4, most, 2048, 1 << 20), (1 << 62, 1 << 10, 64, 2), (4, most, most, most)):
        assert lib.routepack_balance_workspace(_problem(L=L, E=E).ref, T, G) == -8, (T, L, E, G)
    exact = lib.routepack_balance_workspace(_problem(L=most, E=2048).ref, 4, 1 << 16)
    assert exact >= (1 + (1 << 16)) * most * 2048 * 4 + 16 * most * (1 << 16) * 32

    def loss(L, T, G):
        z = _rows(0, T=T, ts=0, ls=0)
        return lib.routepack_balance_loss(_problem(L=L, E=2048).ref, C.byref(z), G, SOME, SOME, 5, 0, SOME, SOME, SOME,
                                          2 ** 62, None)
    assert loss(1 << 20, 4, most) == -8 and loss(1 << 10, 1 << 53, 2) == -8
    for T, L in ((1 << 62, 4), (1 << 40, 1 << 20)):
        z, rec = _rows(0, T=T, ts=0, ls=0), _rows(5, T=T, ts=0, ls=0)
        assert _route(_problem(L=L, E=2048), z) == -8 and _route(_problem(L=L, E=2048), z, rec) == -8
        assert lib.routepack_route_backward(_problem(L=L, E=2048).ref, C.byref(z), C.byref(rec), SOME, 1, 1.0, 0, None,
                                            None, 0, None, 0, SOME, None) == -8
