"""MI355X (gfx950) RoutePack planner hot path -- Python binding.

A thin ctypes layer over the C-ABI in include/routepack.h and, for the
router's operators, include/routepack/router.h (libroutepack.so).
It only marshals arguments (and lets autograd record the router's gates and
loss): torch supplies device memory and the current HIP stream, and every step
of the path runs in the library's HIP kernels.  There is no CPU fallback:
importing works without a GPU, but every call raises if the library or a GPU
is missing.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libroutepack.so")

ERRORS = {0: "ok", -1: "invalid argument", -2: "infeasible window", -3: "FixedRowFFD failed",
          -4: "infeasible layout", -5: "fixed-point overflow", -6: "HIP error",
          -7: "postcondition failed", -8: "unsupported size"}

LEVEL_KERNELS = {0: "workgroup", 1: "wave", 2: "chain", 3: "chain_run"}

EXPORTS = ("routepack_aggregate_demand", "routepack_place_experts", "routepack_pack_rows",
           "routepack_anneal", "routepack_eval_objective", "routepack_select_population",
           "routepack_row_lower_bound", "routepack_fixed_bin_search", "routepack_project_demand",
           "routepack_strerror")
# the router's operators, declared in include/routepack/router.h
ROUTER_EXPORTS = ("routepack_route_tokens", "routepack_count_demand", "routepack_balance_workspace",
                  "routepack_balance_loss", "routepack_route_backward")
# measurement aid declared in include/routepack_probe.h (not part of the method),
# built as its own library
PROBE_EXPORTS = ("routepack_probe_lds_read",)
PROBE_LIB_PATH = os.path.join(_HERE, "libroutepack_probe.so")


class RoutepackError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__(f"{fn} failed: {code} ({ERRORS.get(code, 'unknown')})")
        self.code = code


class _Problem(C.Structure):
    _fields_ = [("n_samples", C.c_int32), ("n_layers", C.c_int32), ("n_experts", C.c_int32),
                ("top_k", C.c_int32), ("n_ranks", C.c_int32), ("n_dp", C.c_int32),
                ("n_edp", C.c_int32), ("dp_to_edp", C.POINTER(C.c_int32)),
                ("capacity", C.c_int64), ("n_stages", C.c_int32),
                ("alpha_fp", C.POINTER(C.c_int64)), ("beta_fp", C.POINTER(C.c_int64)),
                ("frac_bits", C.c_int32), ("min_rows", C.c_int32)]


class _AnnealParams(C.Structure):
    _fields_ = [("n_sweeps", C.c_int32), ("steps_per_sweep", C.c_int32),
                ("temperatures", C.POINTER(C.c_double)), ("t_next", C.c_double),
                ("p_guide_u32", C.c_uint32), ("rho_u32", C.c_uint32), ("seed", C.c_uint64),
                ("sweep_offset", C.c_int32), ("init_incumbent", C.c_int32),
                ("level_kernel_ms", C.POINTER(C.c_double)), ("level_kernel", C.POINTER(C.c_int32))]


class _Rows(C.Structure):
    """routepack_logits and routepack_ids (the same fields)."""
    _fields_ = [("data", C.c_void_p), ("type", C.c_int32), ("n_tokens", C.c_int64), ("token_stride", C.c_int64),
                ("layer_stride", C.c_int64)]


_lib = None


def load_library():
    """Loads libroutepack.so; raises if it was not built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run __graft_entry__.build() first")
        lib = C.CDLL(LIB_PATH)
        vp, i32, i64, u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
        P = C.POINTER(_Problem)
        lib.routepack_aggregate_demand.argtypes = [P, vp, vp, vp]
        lib.routepack_place_experts.argtypes = [P, vp, vp, vp, vp, vp, vp]
        lib.routepack_project_demand.argtypes = [P, vp, vp, vp, vp, vp, vp]
        lib.routepack_pack_rows.argtypes = [P, vp, vp, u64, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        lib.routepack_anneal.argtypes = [P, vp, vp, i32, i32, vp, C.POINTER(_AnnealParams), vp, vp,
                                         vp, vp, vp, vp]
        lib.routepack_eval_objective.argtypes = [P, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.routepack_select_population.argtypes = [P, vp, vp, i32, i32, vp, vp, u64, i32, vp, vp, vp]
        lib.routepack_row_lower_bound.argtypes = [P, vp, C.POINTER(C.c_int32), C.POINTER(C.c_int64), vp]
        lib.routepack_fixed_bin_search.argtypes = [P, vp, i32, i64, C.POINTER(C.c_int32), C.POINTER(C.c_int64), vp,
                                                   vp]
        R, f32 = C.POINTER(_Rows), C.c_float
        lib.routepack_route_tokens.argtypes = [P, R, R, vp, i32, i32, f32, vp, vp, vp]
        lib.routepack_count_demand.argtypes = [P, R, vp, vp, vp]
        lib.routepack_balance_workspace.argtypes = [P, i64, i32]
        lib.routepack_balance_loss.argtypes = [P, R, i32, vp, vp, i32, i32, vp, vp, vp, i64, vp]
        lib.routepack_route_backward.argtypes = [P, R, R, vp, i32, f32, i32, vp, vp, i32, vp, i32, vp, vp]
        lib.routepack_strerror.argtypes = [C.c_int]
        lib.routepack_strerror.restype = C.c_char_p
        for f in EXPORTS:
            if f != "routepack_strerror":
                getattr(lib, f).restype = C.c_int
        for f in ROUTER_EXPORTS:
            getattr(lib, f).restype = C.c_int
        lib.routepack_balance_workspace.restype = C.c_int64
        _lib = lib
    return _lib


class Problem:
    """Problem description (mirrors routepack_problem)."""

    def __init__(self, n_samples, n_layers, n_experts, top_k, n_ranks, n_dp, n_edp, dp_to_edp,
                 capacity, alpha_fp, beta_fp, frac_bits=12, min_rows=1):
        self.dp_to_edp = np.ascontiguousarray(dp_to_edp, dtype=np.int32)
        self.alpha_fp = np.ascontiguousarray(alpha_fp, dtype=np.int64)
        self.beta_fp = np.ascontiguousarray(beta_fp, dtype=np.int64)
        self.n_samples, self.n_layers, self.n_experts = int(n_samples), int(n_layers), int(n_experts)
        self.top_k, self.n_ranks, self.n_dp, self.n_edp = int(top_k), int(n_ranks), int(n_dp), int(n_edp)
        self.capacity, self.frac_bits, self.min_rows = int(capacity), int(frac_bits), int(min_rows)
        self._c = _Problem(self.n_samples, self.n_layers, self.n_experts, self.top_k, self.n_ranks,
                           self.n_dp, self.n_edp,
                           self.dp_to_edp.ctypes.data_as(C.POINTER(C.c_int32)), self.capacity,
                           len(self.alpha_fp), self.alpha_fp.ctypes.data_as(C.POINTER(C.c_int64)),
                           self.beta_fp.ctypes.data_as(C.POINTER(C.c_int64)), self.frac_bits,
                           self.min_rows)

    @classmethod
    def from_dict(cls, d):
        return cls(**d)

    @property
    def ref(self):
        return C.byref(self._c)


def _torch():
    import torch
    if not torch.cuda.is_available():
        raise RuntimeError("the RoutePack HIP path needs a GPU (torch.cuda.is_available() is False)")
    return torch


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    torch = _torch()
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(fn, rc):
    if rc != 0:
        raise RoutepackError(fn, rc)


def _dev(x, dtype):
    torch = _torch()
    if isinstance(x, torch.Tensor):
        assert x.is_cuda and x.dtype == dtype and x.is_contiguous(), (x.device, x.dtype)
        return x
    return torch.as_tensor(np.ascontiguousarray(x), device="cuda").to(dtype).contiguous()


def aggregate_demand(prob: Problem, demand):
    """agg[l][e] = sum_i demand[i][l][e] (int64), computed on the GPU."""
    torch = _torch()
    lib = load_library()
    d = _dev(demand, torch.int32)
    agg = torch.empty((prob.n_layers, prob.n_experts), dtype=torch.int64, device="cuda")
    _check("routepack_aggregate_demand", lib.routepack_aggregate_demand(prob.ref, _ptr(d), _ptr(agg), _stream()))
    return agg


def aggregate_demand_noalloc(prob: Problem, demand, out=None):
    """aggregate_demand through routepack_aggregate_demand_noalloc: the
    library allocates nothing (its partials live in a fixed device array);
    `out` (int64 [L][E] on the device) receives the result when given."""
    torch = _torch()
    lib = load_library()
    d = _dev(demand, torch.int32)
    agg = out if out is not None else torch.empty((prob.n_layers, prob.n_experts), dtype=torch.int64,
                                                  device="cuda")
    _check("routepack_aggregate_demand_noalloc",
           lib.routepack_aggregate_demand_noalloc(prob.ref, _ptr(d), _ptr(agg), _stream()))
    return agg


def place_experts(prob: Problem, agg, demand=None):
    """Layer-local LPT: returns (slot_of [L][E], rank_load [L][P], q [N][L][P] or None)."""
    torch = _torch()
    lib = load_library()
    a = _dev(agg, torch.int64)
    slot = torch.empty((prob.n_layers, prob.n_experts), dtype=torch.int32, device="cuda")
    load = torch.empty((prob.n_layers, prob.n_ranks), dtype=torch.int64, device="cuda")
    d = None if demand is None else _dev(demand, torch.int32)
    q = None
    if d is not None:
        q = torch.empty((prob.n_samples, prob.n_layers, prob.n_ranks), dtype=torch.int32, device="cuda")
    _check("routepack_place_experts", lib.routepack_place_experts(prob.ref, _ptr(a), _ptr(slot), _ptr(load),
                                                                   _ptr(d), _ptr(q), _stream()))
    return slot, load, q


def project_demand(prob: Problem, agg, slot_of, demand=None):
    """A given placement: returns (rank_load [L][P], q [N][L][P] or None)."""
    torch = _torch()
    lib = load_library()
    a = _dev(agg, torch.int64)
    s = _dev(slot_of, torch.int32)
    load = torch.empty((prob.n_layers, prob.n_ranks), dtype=torch.int64, device="cuda")
    d = None if demand is None else _dev(demand, torch.int32)
    q = None
    if d is not None:
        q = torch.empty((prob.n_samples, prob.n_layers, prob.n_ranks), dtype=torch.int32, device="cuda")
    _check("routepack_project_demand", lib.routepack_project_demand(prob.ref, _ptr(a), _ptr(s), _ptr(load),
                                                                     _ptr(d), _ptr(q), _stream()))
    return load, q


def pack_rows(prob: Problem, lengths, q, seed, n_trials, width, pop):
    """Row-count search and seed population; returns a dict."""
    torch = _torch()
    lib = load_library()
    t = _dev(lengths, torch.int32)
    qq = _dev(q, torch.int32)
    popl = torch.empty((pop, prob.n_samples), dtype=torch.int32, device="cuda")
    sc = torch.empty((pop, 3), dtype=torch.int64, device="cuda")
    r_star, cert = C.c_int32(0), C.c_int32(0)
    info = (C.c_int32 * 3)()
    rc = lib.routepack_pack_rows(prob.ref, _ptr(t), _ptr(qq), C.c_uint64(seed), n_trials, width, pop,
                                 C.byref(r_star), C.byref(cert), _ptr(popl), _ptr(sc), info, _stream())
    _check("routepack_pack_rows", rc)
    return dict(r_star=r_star.value, certified=bool(cert.value), population=popl, scores=sc,
                r_lb=info[0], n_distinct=info[1], n_trials_ok=info[2])


def anneal(prob: Problem, lengths, q, n_rows, population, temperatures, steps_per_sweep, seed,
           t_next=0.0, sweep_offset=0, p_guide_u32=0xCCCCCCCD, rho_u32=0x40000000,
           best_layout=None, best_score=None, want_trace=True, want_parents=True, want_steps=False,
           inplace=False, kernel_times=False):
    """Population annealing; returns dict(population, best_layout, best_score, trace, parents, steps)."""
    torch = _torch()
    lib = load_library()
    t = _dev(lengths, torch.int32)
    qq = _dev(q, torch.int32)
    popl = _dev(population, torch.int32)
    if not inplace:
        popl = popl.clone()
    P, N = popl.shape
    temps = np.ascontiguousarray(temperatures, dtype=np.float64)
    ns = len(temps)
    init = best_layout is None
    bl = torch.zeros(N, dtype=torch.int32, device="cuda") if init else _dev(best_layout, torch.int32).clone()
    bs = torch.zeros(3, dtype=torch.int64, device="cuda") if init else _dev(best_score, torch.int64).clone()
    trace = torch.empty((ns, P, 8), dtype=torch.int64, device="cuda") if want_trace else None
    parents = torch.empty((ns, P), dtype=torch.int32, device="cuda") if want_parents else None
    steps = torch.empty((ns, P, steps_per_sweep), dtype=torch.uint8, device="cuda") if want_steps else None
    kms = np.zeros(max(ns, 1), dtype=np.float64) if kernel_times else None
    used = C.c_int32(-1)
    ap = _AnnealParams(ns, steps_per_sweep, temps.ctypes.data_as(C.POINTER(C.c_double)), float(t_next),
                       p_guide_u32, rho_u32, seed, sweep_offset, 1 if init else 0,
                       kms.ctypes.data_as(C.POINTER(C.c_double)) if kms is not None else None,
                       C.pointer(used))
    rc = lib.routepack_anneal(prob.ref, _ptr(t), _ptr(qq), n_rows, P, _ptr(popl), C.byref(ap), _ptr(bl),
                              _ptr(bs), _ptr(trace), _ptr(parents), _ptr(steps), _stream())
    _check("routepack_anneal", rc)
    return dict(population=popl, best_layout=bl, best_score=bs, trace=trace, parents=parents, steps=steps,
                level_kernel_ms=None if kms is None else kms[:ns],
                level_kernel=LEVEL_KERNELS.get(used.value))


def eval_objective(prob: Problem, lengths, q, n_rows, layouts, rank_load=None, want_J=False,
                   want_diag=False):
    """Exact scores, status and optional J / diagnostics of many layouts."""
    torch = _torch()
    lib = load_library()
    t = _dev(lengths, torch.int32)
    qq = _dev(q, torch.int32)
    lay = _dev(layouts, torch.int32)
    if lay.dim() == 1:
        lay = lay.unsqueeze(0)
    n = lay.shape[0]
    sc = torch.empty((n, 3), dtype=torch.int64, device="cuda")
    st = torch.empty(n, dtype=torch.int32, device="cuda")
    J = torch.empty((n, n_rows * prob.n_edp), dtype=torch.int64, device="cuda") if want_J else None
    dg = torch.empty((n, 8), dtype=torch.float64, device="cuda") if want_diag else None
    rl = None if rank_load is None else _dev(rank_load, torch.int64)
    rc = lib.routepack_eval_objective(prob.ref, _ptr(t), _ptr(qq), n_rows, n, _ptr(lay), _ptr(sc), _ptr(st),
                                      _ptr(J), _ptr(dg), _ptr(rl), _stream())
    _check("routepack_eval_objective", rc)
    return dict(scores=sc, status=st, J=J, diag=dg)


_probe_lib = None


def load_probe_library():
    """Loads libroutepack_probe.so (the LDS read-bandwidth probe)."""
    global _probe_lib
    if _probe_lib is None:
        if not os.path.exists(PROBE_LIB_PATH):
            raise RuntimeError(f"{PROBE_LIB_PATH} is missing: run __graft_entry__.build() first")
        lib = C.CDLL(PROBE_LIB_PATH)
        lib.routepack_probe_lds_read.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_double),
                                                 C.POINTER(C.c_int64), C.c_void_p]
        lib.routepack_probe_lds_read.restype = C.c_int
        _probe_lib = lib
    return _probe_lib


def probe_lds_read(n_workgroups=2048, reps=8192):
    """LDS read bandwidth of this device (routepack_probe_lds_read): returns
    (bytes read, launch ms).  A measurement aid, not part of the method."""
    torch = _torch()
    lib = load_probe_library()
    sink = torch.empty(n_workgroups * 256, dtype=torch.int32, device="cuda")
    ms, nbytes = C.c_double(0.0), C.c_int64(0)
    _check("routepack_probe_lds_read",
           lib.routepack_probe_lds_read(int(n_workgroups), int(reps), _ptr(sink), C.byref(ms), C.byref(nbytes),
                                        _stream()))
    return int(nbytes.value), float(ms.value)


def select_population(prob: Problem, lengths, q, n_rows, candidates, primary, seed, pop_size=0):
    """QualityDiversitySelect (routepack_select_population): the selection
    order of the candidates and, when pop_size > 0, the population they fill."""
    torch = _torch()
    lib = load_library()
    t = _dev(lengths, torch.int32)
    qq = _dev(q, torch.int32) if q is not None else None
    cand = _dev(candidates, torch.int32)
    s0 = _dev(primary, torch.int64)
    M = cand.shape[0]
    order = torch.empty(M, dtype=torch.int32, device="cuda")
    pop = torch.empty((pop_size, prob.n_samples), dtype=torch.int32, device="cuda") if pop_size > 0 else None
    _check("routepack_select_population",
           lib.routepack_select_population(prob.ref, _ptr(t), _ptr(qq), int(n_rows), int(M), _ptr(cand), _ptr(s0),
                                           C.c_uint64(seed), int(pop_size), _ptr(order), _ptr(pop), _stream()))
    return {"order": order, "population": pop}


def row_lower_bound(prob: Problem, lengths):
    """(R_bound, K_bound) of routepack_row_lower_bound: R* is minimal when it
    equals R_bound."""
    torch = _torch()
    lib = load_library()
    t = _dev(lengths, torch.int32)
    r, k = C.c_int32(0), C.c_int64(0)
    _check("routepack_row_lower_bound", lib.routepack_row_lower_bound(prob.ref, _ptr(t), C.byref(r), C.byref(k),
                                                                      _stream()))
    return int(r.value), int(k.value)


def fixed_bin_search(prob: Problem, lengths, n_rows, node_budget):
    """routepack_fixed_bin_search: (status, nodes, layout or None); status 1
    feasible, 0 infeasible, 2 unknown."""
    torch = _torch()
    lib = load_library()
    t = _dev(lengths, torch.int32)
    lay = torch.full((prob.n_samples,), -1, dtype=torch.int32, device="cuda")
    st, nodes = C.c_int32(0), C.c_int64(0)
    _check("routepack_fixed_bin_search",
           lib.routepack_fixed_bin_search(prob.ref, _ptr(t), int(n_rows), int(node_budget), C.byref(st),
                                          C.byref(nodes), _ptr(lay), _stream()))
    return int(st.value), int(nodes.value), (lay if st.value == 1 else None)


# -- the router's operators (include/routepack/router.h) ----------------------

SCORES = {"softmax": 0, "sigmoid": 1}


_ROUTER = None


def _router():
    """(the library, torch, types of logits, types of ids), looked up once:
    the smallest calls take a few microseconds."""
    global _ROUTER
    if _ROUTER is None:
        lib, torch = load_library(), _torch()
        _ROUTER = (lib, torch, {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2},
                   {torch.uint8: 3, torch.int16: 4, torch.int32: 5, torch.int64: 6})
    return _ROUTER


def _raw_stream(device):
    """The current stream's handle (without a torch.cuda.Stream object where
    torch offers that)."""
    torch = _ROUTER[1]
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw is not None else torch.cuda.current_stream(device).cuda_stream


class _Call:
    """One call's tensors: checks that they share a GPU, hands out pointers,
    and runs the call on that GPU's current stream."""

    __slots__ = ("fn", "torch", "device")

    def __init__(self, fn, torch):
        self.fn, self.torch, self.device = fn, torch, None

    def tensor(self, name, x, dtypes, shape=None):
        if not isinstance(x, self.torch.Tensor):
            raise TypeError(f"{self.fn}: {name} must be a tensor, got {type(x).__name__}")
        if not x.is_cuda or (self.device is not None and x.device != self.device):
            raise ValueError(f"{self.fn}: {name} is on {x.device}, expected {self.device or 'a GPU'}")
        if self.device is None:
            self.device = x.device
        if x.dtype not in dtypes:
            raise ValueError(f"{self.fn}: {name} has type {x.dtype}")
        if shape is not None and tuple(x.shape) != tuple(shape):
            raise ValueError(f"{self.fn}: {name} has shape {tuple(x.shape)}, expected {tuple(shape)}")
        return x

    def dense(self, name, x, dtypes, shape):
        x = self.tensor(name, x, dtypes, shape)
        if not x.is_contiguous():
            raise ValueError(f"{self.fn}: {name} must be contiguous")
        return x

    def rows(self, name, x, dtypes, L, last):
        """[T][L][last], or [T][last] where L is 1, of any strides but the
        last: (the tensor's shape, its description for the library)."""
        self.tensor(name, x, dtypes)
        shape, stride = x.shape, x.stride()
        three = len(shape) == 3
        if not (three and shape[1] == L or len(shape) == 2 and L == 1) or shape[-1] != last:
            raise ValueError(f"{self.fn}: {name} has shape {tuple(shape)}, expected [T][{L}][{last}]")
        if last > 1 and stride[-1] != 1 and shape[0] > 0:
            raise ValueError(f"{self.fn}: the last axis of {name} must be adjacent in memory")
        return shape, _Rows(x.data_ptr(), dtypes[x.dtype], shape[0], stride[0], stride[1] if three else 0)

    def run(self, f, *args):
        cuda = self.torch.cuda
        stream = _raw_stream(self.device)
        if self.device.index == cuda.current_device():
            rc = f(*args, stream)
        else:
            with cuda.device(self.device):
                rc = f(*args, stream)
        if rc != 0:
            raise RoutepackError(self.fn, rc)


def _score(fn, score):
    if score not in SCORES:
        raise ValueError(f"{fn}: score is {score!r}, expected one of {sorted(SCORES)}")
    return SCORES[score]


_FUNCTIONS = None


def _functions():
    """(gates, loss) as functions that autograd records: route_tokens and
    balance_loss go through them, and they (with recording off) through these,
    where the logits require a gradient.  Their backward passes are
    route_backward's; ids and counts are constants."""
    global _FUNCTIONS
    if _FUNCTIONS is not None:
        return _FUNCTIONS
    torch = _router()[1]
    once_differentiable = torch.autograd.function.once_differentiable

    class Gates(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, prob, ids, bias, score, normalize, scale):
            out, gates = route_tokens(prob, logits, ids=ids, bias=bias, score=score, normalize=normalize, scale=scale)
            ctx.save_for_backward(logits, out)
            ctx.set_materialize_grads(False)
            ctx.args = prob, dict(score=score, normalize=normalize, scale=scale)
            if ids is not None:
                return gates
            ctx.mark_non_differentiable(out)
            return out, gates

        @staticmethod
        @once_differentiable
        def backward(ctx, *grads):
            dz = None
            if grads[-1] is not None:
                (logits, ids), (prob, how) = ctx.saved_tensors, ctx.args
                dz = route_backward(prob, logits, ids=ids, dgates=grads[-1].contiguous(), **how)
            return dz, None, None, None, None, None, None

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, prob, counts, offsets, score):
            ctx.save_for_backward(logits, counts, offsets)
            ctx.set_materialize_grads(False)
            ctx.args = prob, score
            return balance_loss(prob, logits, counts, offsets, score=score)

        @staticmethod
        @once_differentiable
        def backward(ctx, dloss, dshares):
            if dshares is not None:
                raise NotImplementedError("routepack_balance_loss: the shares have no gradient, only the loss has")
            dz = None
            if dloss is not None:
                (logits, counts, offsets), (prob, score) = ctx.saved_tensors, ctx.args
                dz = route_backward(prob, logits, counts=counts, offsets=offsets, dloss=dloss.contiguous(),
                                    score=score)
            return dz, None, None, None, None

    _FUNCTIONS = Gates, Loss
    return _FUNCTIONS


def route_tokens(prob: Problem, logits, *, ids=None, bias=None, score="softmax", normalize=True, scale=1.0):
    """The router's gates: (ids, gates), each [T][L][k] (or [T][k] for logits
    [T][E]), k = prob.top_k.

    logits [T][L][E] fp32, bf16 or fp16, any strides over tokens and layers.
    Without `ids` the k experts of largest logit are chosen, or, with `bias`
    (float32 [L][E]), of largest score + bias; ids are int32, -1 where no
    expert is available (an expert is masked by a logit of -inf).  With `ids`
    (uint8, int16, int32 or int64; a replayed record) the gates are those of
    the recorded experts, and `ids` is returned as it is.  score: "softmax"
    or "sigmoid"; normalize: divide by the sum over the token's choices.

    Where the logits require a gradient, autograd records the gates: their
    backward pass is route_backward's with the ids as constants (none reaches
    the bias, which takes no part in the gates).  A trainer that has the
    gradients of gates and loss at hand saves a pass by calling route_backward
    itself, under torch.no_grad().  (As for all that autograd records: before a
    backward pass is captured into a graph, results recorded eagerly from the
    same leaves are to be released.)"""
    lib, torch, floats, ints = _router()
    call = _Call("routepack_route_tokens", torch)
    shape, z = call.rows("logits", logits, floats, prob.n_layers, prob.n_experts)
    if logits.requires_grad and torch.is_grad_enabled():
        out = _functions()[0].apply(logits, prob, ids, bias, score, normalize, scale)
        return out if ids is None else (ids, out)
    shape = (*shape[:-1], prob.top_k)
    b = bias
    if bias is not None:
        b = call.dense("bias", bias, (torch.float32,), (prob.n_layers, prob.n_experts)).data_ptr()
    out, rec = ids, None
    if ids is not None:
        got, rec = call.rows("ids", ids, ints, prob.n_layers, prob.top_k)
        if tuple(got) != shape:
            raise ValueError(f"{call.fn}: ids has shape {tuple(got)}, expected {shape}")
        rec = C.byref(rec)
    else:
        out = torch.empty(shape, dtype=torch.int32, device=call.device)
    gates = torch.empty(shape, dtype=torch.float32, device=call.device)
    call.run(lib.routepack_route_tokens, prob.ref, C.byref(z), rec, b, _score(call.fn, score), 1 if normalize else 0,
             scale, out.data_ptr() if ids is None else None, gates.data_ptr())
    return out, gates


def count_demand(prob: Problem, ids, offsets):
    """demand int32 [N][L][E]: how often each sample's tokens chose each
    expert, the `demand` of aggregate_demand and place_experts.

    ids [T][L][k] (or [T][k] where L is 1) uint8, int16, int32 or int64, any
    strides over tokens and layers; ids outside [0, E) are not counted.
    offsets int64 [N + 1], non-decreasing: sample i holds the tokens
    [offsets[i], offsets[i + 1])."""
    lib, torch, _, ints = _router()
    call = _Call("routepack_count_demand", torch)
    _, x = call.rows("ids", ids, ints, prob.n_layers, prob.top_k)
    off = call.dense("offsets", offsets, (torch.int64,), (prob.n_samples + 1,))
    demand = torch.empty((prob.n_samples, prob.n_layers, prob.n_experts), dtype=torch.int32, device=call.device)
    call.run(lib.routepack_count_demand, prob.ref, C.byref(x), off.data_ptr(), demand.data_ptr())
    return demand


def _groups(call, prob, counts, offsets):
    _, torch, _, ints = _router()
    off = call.tensor("offsets", offsets, (torch.int64,))
    if off.dim() != 1 or off.shape[0] < 2 or not off.is_contiguous():
        raise ValueError(f"{call.fn}: offsets has shape {tuple(off.shape)}, expected [G + 1], contiguous, with G >= 1")
    G = off.shape[0] - 1
    n = call.dense("counts", counts, (torch.int32, torch.int64), (G, prob.n_layers, prob.n_experts))
    return G, off.data_ptr(), n.data_ptr(), ints[n.dtype]


def balance_loss(prob: Problem, logits, counts, offsets, *, score="softmax"):
    """The balance loss: (loss float32 [L], shares float32 [G][L][E]).

    loss[l] = 1/G sum_g sum_e f[g][l][e] shares[g][l][e] with f the fraction of
    the counts that expert e has, times E, and shares the mean over the
    group's tokens of the scores divided by their sum.  counts int32 or int64
    [G][L][E] (count_demand's result, or aggregate_demand's as [1][L][E] for
    one group over the window); offsets int64 [G + 1].

    Where the logits require a gradient, autograd records the loss: its
    backward pass is route_backward's with the counts as constants.  The
    shares' own gradient is not formed; a backward pass through them raises."""
    lib, torch, floats, _ = _router()
    call = _Call("routepack_balance_loss", torch)
    shape, z = call.rows("logits", logits, floats, prob.n_layers, prob.n_experts)
    if logits.requires_grad and torch.is_grad_enabled():
        return _functions()[1].apply(logits, prob, counts, offsets, score)
    G, off, n, n_type = _groups(call, prob, counts, offsets)
    L, E, at = prob.n_layers, prob.n_experts, call.device
    loss = torch.empty(L, dtype=torch.float32, device=at)
    shares = torch.empty((G, L, E), dtype=torch.float32, device=at)
    size = lib.routepack_balance_workspace(prob.ref, shape[0], G)
    work = torch.empty(max(size, 16), dtype=torch.uint8, device=at)
    call.run(lib.routepack_balance_loss, prob.ref, C.byref(z), G, off, n, n_type, _score(call.fn, score),
             loss.data_ptr(), shares.data_ptr(), work.data_ptr(), size)
    return loss, shares


def route_backward(prob: Problem, logits, *, ids=None, dgates=None, normalize=True, scale=1.0, counts=None,
                   offsets=None, dloss=None, score="softmax"):
    """dlogits, of the logits' shape and type, from the gradients of
    route_tokens' gates (`ids`, `dgates` float32 of their shape, `normalize`,
    `scale`), of balance_loss' loss (`counts`, `offsets`, `dloss` float32 [L]),
    or of both in one pass.  The result itself carries no gradient."""
    lib, torch, floats, ints = _router()
    call = _Call("routepack_route_backward", torch)
    if (ids is None) != (dgates is None):
        raise ValueError(f"{call.fn}: ids and dgates go together")
    if (dloss is None) != (counts is None) or (dloss is None) != (offsets is None):
        raise ValueError(f"{call.fn}: counts, offsets and dloss go together")
    if ids is None and dloss is None:
        raise ValueError(f"{call.fn}: neither dgates nor dloss given")
    shape, z = call.rows("logits", logits, floats, prob.n_layers, prob.n_experts)
    rec = dg = off = n = dl = None
    G = n_type = 0
    if ids is not None:
        got, rec = call.rows("ids", ids, ints, prob.n_layers, prob.top_k)
        if got[:-1] != shape[:-1]:
            raise ValueError(f"{call.fn}: ids has shape {tuple(got)}, logits {tuple(shape)}")
        dg = call.dense("dgates", dgates, (torch.float32,), got).data_ptr()
        rec = C.byref(rec)
    if dloss is not None:
        G, off, n, n_type = _groups(call, prob, counts, offsets)
        dl = call.dense("dloss", dloss, (torch.float32,), (prob.n_layers,)).data_ptr()
    dz = torch.empty(shape, dtype=logits.dtype, device=call.device)
    call.run(lib.routepack_route_backward, prob.ref, C.byref(z), rec, dg, 1 if normalize else 0, scale, G, off, n,
             n_type, dl, _score(call.fn, score), dz.data_ptr())
    return dz
