"""Host-side checks of the experts' entry points (include/routepack/experts.h)
and of the router's grouped choice that need no GPU, and pins of their oracle:
argument errors come before any device work, and the oracle's formulas agree
with small worked examples."""
import ctypes as C
import os
import re

import numpy as np

from oracle import experts as X

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOME = C.c_void_p(64)  # never read: every call below is refused, or has no work


def _problem(N=2, L=3, E=16, k=2):
    import paper_2608_12146_amd as rp
    return rp.Problem(N, L, E, k, 1, 1, 1, [0], 64, [1], [0])


def _rows(type_=5, T=4, data=64, ts=48, ls=16):
    import paper_2608_12146_amd as rp
    return rp._Rows(data, type_, T, ts, ls)


def _matrix(rows=4, cols=40, type_=1, stride=None, data=64):
    import paper_2608_12146_amd as rp
    return rp._MATRIX(data or 0, type_, rows, cols, cols if stride is None else stride)


def _mx(rows=4, cols=40, codes=64, scales=64):
    import paper_2608_12146_amd as rp
    return rp._MX(codes or 0, scales or 0, rows, cols)


def _by(x):
    return x if x is None or isinstance(x, bytes) else C.byref(x)


def test_every_declared_entry_point_is_exported():
    import paper_2608_12146_amd as rp
    src = open(os.path.join(ROOT, "include", "routepack", "experts.h")).read()
    names = re.findall(r"^(?:int|int64_t)\s+(routepack_\w+)\s*\(", src, re.M)
    assert sorted(names) == sorted(rp.EXPERT_EXPORTS)
    lib = rp.load_library()
    assert all(hasattr(lib, n) for n in names)


def test_grouped_route_refusals():
    import paper_2608_12146_amd as rp

    def call(prob, z, bias=None, groups=4, keep=2, top=1, score=0, scale=1.0, ids=SOME, gates=SOME):
        return rp.load_library().routepack_route_grouped(prob and prob.ref, _by(z), bias, groups, keep, top, score, 1,
                                                         scale, ids, gates, None)
    F = _rows(0)
    assert call(None, F) == -1 and call(_problem(), None) == -1
    for bad in (_rows(3), _rows(0, T=-1), _rows(0, data=None), _rows(0, ts=-1)):
        assert call(_problem(), bad) == -1
    for more in (dict(groups=0), dict(groups=3), dict(groups=32), dict(keep=0), dict(keep=5), dict(top=0), dict(top=3),
                 dict(score=2), dict(scale=float("nan")), dict(ids=None), dict(gates=None)):
        assert call(_problem(), F, **more) == -1, more
    assert call(_problem(k=9), F) == -1 and call(_problem(k=8), F, ids=None) == -1
    assert call(_problem(E=1028), F) == -8 and call(_problem(E=130), F, groups=65) == -8
    assert call(_problem(E=256, k=33), F, keep=4) == -8
    assert call(_problem(), _rows(0, T=0, data=None), ids=None, gates=None) == 0


def test_order_refusals():
    import paper_2608_12146_amd as rp
    lib = rp.load_library()

    def call(prob, ids, rows=SOME, off=SOME, places=SOME, work=SOME, size=1 << 40):
        return lib.routepack_order_tokens(prob and prob.ref, _by(ids), None, rows, off, places, work, size, None)
    I = _rows()
    assert call(None, I) == -1 and call(_problem(), None) == -1
    for bad in (_rows(0), _rows(7), _rows(T=-1), _rows(data=None), _rows(ts=-1), _rows(ls=-1)):
        assert call(_problem(), bad) == -1
    many = _rows(T=1 << 20)
    for more in (dict(rows=None), dict(off=None), dict(places=None), dict(work=None), dict(work=C.c_void_p(72)), dict(size=8)):
        assert call(_problem(), many, **more) == -1, more
    assert call(_problem(E=0), I) == -1 and call(_problem(k=0), I) == -1 and call(_problem(L=-1), I) == -1
    assert call(_problem(E=2049), I) == -8 and call(_problem(k=257), I) == -8
    assert call(_problem(), _rows(T=1 << 30)) == -8
    need = lib.routepack_order_workspace(_problem().ref, 1 << 20)
    assert lib.routepack_order_workspace(_problem().ref, 64) == 0
    assert need > 16 and call(_problem(), _rows(T=1 << 20), size=need - 1) == -1
    assert lib.routepack_order_workspace(None, 4) == -1 and lib.routepack_order_workspace(_problem().ref, -1) == -1
    assert call(_problem(L=0), I, None, None, None, None, 0) == 0


def test_mx_refusals():
    import paper_2608_12146_amd as rp
    lib = rp.load_library()

    def quant(x, q, rows=None, places=None, k=2):
        return lib.routepack_quantize_mx(_by(x), rows, _by(places), k, _by(q), None)

    def back(q, x):
        return lib.routepack_dequantize_mx(_by(q), _by(x), None)
    for x in (None, _matrix(type_=3), _matrix(rows=-1), _matrix(cols=-1), _matrix(stride=-1), _matrix(data=None),
              _matrix(rows=5), _matrix(cols=41)):
        assert quant(x, _mx()) == -1 and back(_mx(), x) == -1
    for q in (None, _mx(rows=-1), _mx(cols=-1), _mx(codes=None), _mx(scales=None), _mx(codes=72), _mx(scales=66)):
        assert quant(_matrix(), q) == -1 and back(q, _matrix()) == -1
    assert quant(_matrix(), _mx(8), SOME, None) == -1 and quant(_matrix(), _mx(8), None, _rows()) == -1
    for bad in (_rows(6), _rows(T=5), _rows(ts=-1), _rows(data=None)):
        assert quant(_matrix(), _mx(8), SOME, bad) == -1
    assert quant(_matrix(), _mx(8), SOME, _rows(), k=0) == -1 and quant(_matrix(), _mx(8), SOME, _rows(), k=257) == -8
    assert quant(_matrix(rows=1 << 30), _mx(8), SOME, _rows(T=1 << 30)) == -8
    assert quant(_matrix(), _mx(0, codes=None, scales=None), None, _rows()) == 0
    assert back(_mx(), _matrix(stride=41)) == -1
    big = (1 << 24) + 1
    assert quant(_matrix(cols=big), _mx(cols=big)) == -8
    assert quant(_matrix(rows=1 << 50, cols=1 << 20), _mx(1 << 50, 1 << 20)) == -8
    assert quant(_matrix(rows=0, data=None), _mx(rows=0, codes=None, scales=None)) == 0
    assert back(_mx(cols=0, codes=None, scales=None), _matrix(cols=0, data=None)) == 0


def test_product_refusals():
    import paper_2608_12146_amd as rp
    lib = rp.load_library()

    def call(x, w, n=3, off=SOME, y=None):
        return lib.routepack_expert_product(_by(x), _by(w), n, off, _by(y), None)
    x, w, y = _mx(), _mx(rows=15), _matrix(cols=5)
    for bad in (None, _mx(rows=-1), _mx(cols=41), _mx(codes=None), _mx(scales=9), _mx(rows=5)):
        assert call(bad, w, y=y) == -1
    for bad in (None, _mx(rows=16), _mx(rows=15, cols=39), _mx(rows=15, codes=65)):
        assert call(x, bad, y=y) == -1
    for bad in (None, _matrix(cols=6), _matrix(rows=3, cols=5), _matrix(cols=5, type_=4), _matrix(cols=5, stride=6),
                _matrix(cols=5, data=None)):
        assert call(x, w, y=bad) == -1
    assert call(x, w, n=0, y=y) == -1 and call(x, w, off=None, y=y) == -1
    assert call(x, _mx(rows=2049), n=2049, y=_matrix(cols=1)) == -8
    assert call(_mx(rows=0), w, y=_matrix(rows=0, cols=5, data=None)) == 0

    def grad(dy, x, w, n=3, off=SOME, dx=None, dw=None):
        return lib.routepack_expert_product_backward(_by(dy), _by(x), _by(w), n, off, _by(dx), _by(dw), None)
    dy, dx, dw = _matrix(cols=5), _matrix(), _matrix(rows=15)
    assert grad(dy, x, w) == -1
    for bad in (None, _matrix(cols=4), _matrix(rows=5, cols=5), _matrix(cols=5, type_=3), _matrix(cols=5, stride=-1)):
        assert grad(bad, x, w, dx=dx, dw=dw) == -1
    assert grad(dy, _mx(codes=None), w, dw=dw) == -1 and grad(dy, x, _mx(rows=15, codes=None), dx=dx) == -1
    for bad in (_matrix(type_=0), _matrix(rows=5), _matrix(stride=41), _matrix(data=None)):
        assert grad(dy, x, w, dx=bad) == -1
    for bad in (_matrix(rows=15, type_=0), _matrix(rows=14), _matrix(rows=15, data=None)):
        assert grad(dy, x, w, dw=bad) == -1
    assert grad(dy, x, w, off=None, dx=dx) == -1 and grad(dy, x, w, n=0, dx=dx) == -1
    assert grad(dy, x, _mx(rows=2049), n=2049, dx=dx) == -1  # (dy has other columns)
    assert grad(_matrix(cols=1), x, _mx(rows=2049), n=2049, dx=dx) == -8


def test_combine_refusals():
    import paper_2608_12146_amd as rp
    lib = rp.load_library()

    def call(y, p, k=2, gates=SOME, gs=2, out=None):
        return lib.routepack_combine_tokens(_by(y), _by(p), k, gates, gs, _by(out), None)
    y, p, out = _matrix(rows=8), _rows(), _matrix()
    for bad in (None, _matrix(rows=-1), _matrix(rows=8, type_=5), _matrix(rows=8, data=None), _matrix(rows=8, cols=41)):
        assert call(bad, p, out=out) == -1
    for bad in (None, _rows(6), _rows(T=-1), _rows(ts=-1), _rows(data=None), _rows(T=5)):
        assert call(y, bad, out=out) == -1
    for bad in (None, _matrix(type_=0), _matrix(stride=41), _matrix(data=None)):
        assert call(y, p, out=bad) == -1
    assert call(y, p, k=0, out=out) == -1 and call(y, p, gs=-1, out=out) == -1
    assert call(y, p, k=33, out=out) == -8
    assert call(y, _rows(T=1 << 30), out=_matrix(rows=1 << 30)) == -8
    assert call(y, _rows(T=0, data=None), out=_matrix(rows=0, data=None)) == 0

    def grad(dout, y, rows, p, k=2, gates=SOME, dy=None, dgates=None):
        return lib.routepack_combine_backward(_by(dout), _by(y), rows, _by(p), k, gates, 2, _by(dy), dgates, None)
    assert grad(out, y, SOME, p) == -1
    assert grad(out, y, None, p, dy=y) == -1 and grad(out, y, SOME, p, dy=_matrix(rows=7)) == -1
    assert grad(out, y, SOME, p, dy=_matrix(rows=8, type_=2)) == -1
    assert grad(_matrix(rows=5), y, SOME, p, dy=y) == -1 and grad(_matrix(type_=0), y, SOME, p, dy=y) == -1
    assert grad(out, _matrix(rows=8, data=None), SOME, p, dgates=SOME) == -1
    assert grad(out, y, SOME, p, k=33, dgates=SOME) == -8


# -- pins of the oracle -------------------------------------------------------

def test_oracle_groups():
    z = np.log(np.array([[[4.0, 1.0, 3.0, 2.5, 0.5, 6.0]]]))
    assert X.choose_groups(z, 2, 3, 1).tolist() == [[[5, 4]]]       # by the maximum: 4, 3, 6
    assert X.choose_groups(z, 2, 3, 2).tolist() == [[[5, 0]]]
    assert X.choose_groups(z, 3, 3, 2, top=2).tolist() == [[[5, 2, 3]]]  # by two: 5, 5.5, 6.5
    bias = np.array([[0.0, 0.0, 0.0, 0.0, 0.0, -1.0]])
    assert X.choose_groups(z, 3, 3, 2, top=2, bias=bias).tolist() == [[[0, 2, 3]]]
    assert X.choose_groups(np.full((1, 1, 4), -np.inf), 2, 2, 1).tolist() == [[[-1, -1]]]


def test_oracle_order():
    ids = np.array([[[2, 0]], [[-1, 2]], [[1, 5]]])
    rows, off, places = X.order(ids, 3)
    assert rows.tolist() == [[1, 4, 0, 3, -1, -1]] and off.tolist() == [[0, 1, 2, 4]]
    assert places.tolist() == [[[2, 0]], [[-1, 3]], [[1, -1]]]
    rows, off, _ = X.order(ids, 3, np.array([[1, 2, 0]]))
    assert rows.tolist() == [[0, 3, 1, 4, -1, -1]] and off.tolist() == [[0, 2, 3, 4]]


def test_oracle_blocks():
    x = np.zeros((3, 33))
    x[0, :12] = [4.0, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 7.9, -0.0, 0.76]
    x[1, 0], x[1, 32] = np.nan, 2.0 ** -127
    x[2, :2] = 2.0 ** 127, -2.0 ** 125
    codes, scales = X.quantize(x)
    assert codes.shape == (3, 64) and scales[:, :2].tolist() == [[127, 0], [255, 0], [252, 0]]
    got = X.values(codes, scales, 33)
    assert got[0, :12].tolist() == [4.0, -0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0, -0.0, 1.0]
    assert np.isnan(got[1, :32]).all() and got[1, 32] == 2.0 ** -127
    assert got[2, :3].tolist() == [2.0 ** 127, -2.0 ** 125, 0.0]
    # the packed order: the even column in the low half, two's exponent 2 less
    codes, scales = X.quantize(np.array([[1.0, -2.0]]))
    assert codes[0, 0] == (4 + 16 * 14) and scales[0, 0] == 126


# -- the binding without a GPU --------------------------------------------------

class _FakeTensor:
    """As much of a tensor on a GPU as the binding looks at; addresses are its own."""

    next_address = 1 << 20
    is_cuda, requires_grad = True, False

    def __init__(self, shape, dtype, device="gpu"):
        self.shape, self.dtype, self.device = tuple(shape), dtype, device
        self.address = _FakeTensor.next_address
        _FakeTensor.next_address += 1 << 20

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.address


def _without_gpu(monkeypatch, during):
    """Lets the binding run on _FakeTensors: `during` gets a call's name, its
    arguments and the live tensors' addresses, in place of the library."""
    import types
    import weakref

    import torch

    import paper_2608_12146_amd as rp
    live = weakref.WeakValueDictionary()

    def tensor(shape, dtype, device="gpu"):
        x = _FakeTensor((shape,) if isinstance(shape, int) else shape, dtype, device)
        live[x.address] = x
        return x
    names = ("uint8", "int16", "int32", "int64", "float32", "bfloat16", "float16", "is_grad_enabled")
    fake = types.SimpleNamespace(Tensor=_FakeTensor, empty=tensor, **{n: getattr(torch, n) for n in names})
    real = rp.load_library()

    class Library:
        routepack_order_workspace = real.routepack_order_workspace

        def __getattr__(self, name):
            def call(*args):
                during(name, args, dict(live))
                return 0
            return call

    def run(self, f, *args):
        assert f(*args, None) == 0
    floats = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
    ints = {torch.uint8: 3, torch.int16: 4, torch.int32: 5, torch.int64: 6}
    monkeypatch.setattr(rp, "_router", lambda: (Library(), fake, floats, ints))
    monkeypatch.setattr(rp._Call, "run", run)
    return tensor


def test_workspaces_live_through_the_call(monkeypatch):
    """Memory of the binding's own goes back to the allocator after the call's
    kernels stand in the stream: another thread's call on that stream could else
    be given it while they are being launched."""
    import torch

    import paper_2608_12146_amd as rp
    seen = []

    def during(name, args, live):
        # rows, offsets, places and the workspace of routepack_order_tokens
        seen.append((name, args[7], [a in live for a in args[3:7]]))
    tensor = _without_gpu(monkeypatch, during)
    rp.order_tokens(_problem(L=1, E=256, k=8), tensor((9000, 1, 8), torch.int32))
    (name, size, alive), = seen
    assert name == "routepack_order_tokens" and size > 0
    assert alive == [True] * 4
