"""MI355X (gfx950) RoutePack planner hot path -- Python binding.

A thin ctypes layer over the C-ABI in include/routepack.h and, for the
router's and the experts' operators, include/routepack/router.h and experts.h
(libroutepack.so).  It only marshals arguments (and lets autograd record the
router's gates and loss, quantized matrices, the experts' products and their
sums, in reverse mode): torch supplies device memory and the current HIP stream,
and every step of the path runs in the library's HIP kernels.  There is no CPU
fallback: importing works without a GPU, but every call raises if the library or
a GPU is missing.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

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
ROUTER_EXPORTS = ("routepack_route_tokens", "routepack_route_grouped", "routepack_count_demand", "routepack_balance_workspace",
                  "routepack_balance_loss", "routepack_route_backward")
# the experts' operators, declared in include/routepack/experts.h
EXPERT_EXPORTS = ("routepack_order_workspace", "routepack_order_tokens", "routepack_quantize_mx",
                  "routepack_dequantize_mx", "routepack_expert_product", "routepack_expert_product_backward",
                  "routepack_combine_tokens", "routepack_combine_backward")
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
        lib.routepack_route_grouped.argtypes = [P, R, vp, i32, i32, i32, i32, i32, f32, vp, vp, vp]
        M = X = vp  # (routepack_matrix, routepack_mx and routepack_ids, also as packed bytes)
        lib.routepack_order_workspace.argtypes = [P, i64]
        lib.routepack_order_tokens.argtypes = [P, R, vp, vp, vp, vp, vp, i64, vp]
        lib.routepack_quantize_mx.argtypes = [M, vp, vp, i32, X, vp]
        lib.routepack_dequantize_mx.argtypes = [X, M, vp]
        lib.routepack_expert_product.argtypes = [X, X, i32, vp, M, vp]
        lib.routepack_expert_product_backward.argtypes = [M, X, X, i32, vp, M, M, vp]
        lib.routepack_combine_tokens.argtypes = [M, vp, i32, vp, i64, M, vp]
        lib.routepack_combine_backward.argtypes = [M, M, vp, vp, i32, vp, i64, M, vp, vp]
        lib.routepack_strerror.argtypes = [C.c_int]
        lib.routepack_strerror.restype = C.c_char_p
        for f in EXPORTS:
            if f != "routepack_strerror":
                getattr(lib, f).restype = C.c_int
        for f in ROUTER_EXPORTS + EXPERT_EXPORTS:
            getattr(lib, f).restype = C.c_int
        lib.routepack_balance_workspace.restype = C.c_int64
        lib.routepack_order_workspace.restype = C.c_int64
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
_FORWARD = None  # torch.autograd.forward_ad


def _router():
    """(the library, torch, types of logits, types of ids), looked up once:
    the smallest calls take a few microseconds."""
    global _ROUTER, _FORWARD
    if _ROUTER is None:
        lib, torch = load_library(), _torch()
        _FORWARD = torch.autograd.forward_ad
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
        # (outside of forward mode the level is below 0; where torch hides it, each tensor is asked)
        if _FORWARD is not None and getattr(_FORWARD, "_current_level", 0) >= 0 and _FORWARD.unpack_dual(x).tangent is not None:
            raise NotImplementedError(f"{self.fn}: {name} has a tangent; gradients are formed in reverse mode alone")
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
        def forward(ctx, logits, prob, ids, bias, score, normalize, scale, groups, keep, group_top):
            out, gates = route_tokens(prob, logits, ids=ids, bias=bias, score=score, normalize=normalize, scale=scale,
                                      groups=groups, keep=keep, group_top=group_top)
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
            return (dz,) + (None,) * 9

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


def route_tokens(prob: Problem, logits, *, ids=None, bias=None, score="softmax", normalize=True, scale=1.0, groups=None,
                 keep=None, group_top=1):
    """The router's gates: (ids, gates), each [T][L][k] (or [T][k] for logits
    [T][E]), k = prob.top_k.

    logits [T][L][E] fp32, bf16 or fp16, any strides over tokens and layers.
    Without `ids` the k experts of largest logit are chosen, or, with `bias`
    (float32 [L][E]), of largest score + bias; ids are int32, -1 where no
    expert is available (an expert is masked by a logit of -inf).  With `ids`
    (uint8, int16, int32 or int64; a replayed record) the gates are those of
    the recorded experts, and `ids` is returned as it is.  score: "softmax"
    or "sigmoid"; normalize: divide by the sum over the token's choices.

    With `groups` (not with `ids`) the choice is among the experts of the
    `keep` best of that many groups of adjacent experts, by the sum of each
    group's `group_top` (1 or 2) largest keys, which are the scores with the
    bias added.

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
        out = _functions()[0].apply(logits, prob, ids, bias, score, normalize, scale, groups, keep, group_top)
        return out if ids is None else (ids, out)
    if (groups is None) != (keep is None):
        raise ValueError(f"{call.fn}: groups and keep go together")
    if groups is not None and ids is not None:
        raise ValueError(f"{call.fn}: recorded ids are not chosen among groups")
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
    if groups is not None:
        call.fn = "routepack_route_grouped"
        call.run(lib.routepack_route_grouped, prob.ref, C.byref(z), b, groups, keep, group_top, _score(call.fn, score),
                 1 if normalize else 0, scale, out.data_ptr(), gates.data_ptr())
        return out, gates
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


# -- the experts' operators (include/routepack/experts.h) ----------------------

class Order:
    """The order of (token, choice) pairs by slot, of order_tokens: pair t k + j
    is token t's choice j.

    rows    int32 [P], P = T k: the pair in each row, -1 behind the last one made
    offsets int64 [E + 1]: slot s has the rows [offsets[s], offsets[s + 1])
    places  int32 [T][k]: the row of each pair, -1 where no choice was made

    For L layers rows is [L][P], offsets [L][E + 1] and places [T][L][k]; `layer`
    gives one layer's, which is what the other operators take."""

    __slots__ = ("rows", "offsets", "places")

    def __init__(self, rows, offsets, places):
        self.rows, self.offsets, self.places = rows, offsets, places

    def layer(self, l):
        if self.rows.dim() != 2:
            raise ValueError("this Order is one layer's")
        return Order(self.rows[l], self.offsets[l], self.places[:, l])


class Mx:
    """A matrix [...][rows][columns] in microscaled 4-bit floating point (OCP
    MXFP4): blocks of 32 columns with a common power of two.

    codes  uint8 [...][rows][64 n], n = ceil(columns / 128): two values a byte, the
           even column in the low half; sign, two bits of exponent, one of mantissa
    scales uint8 [...][rows][4 n]: the blocks' exponents plus 127, 255 for NaN

    Columns behind the last are zero codes with scale 0.  What quantize_mx made
    of a tensor that requires a gradient leads autograd back to it (`link`, a
    tensor of this shape whose values mean nothing); other matrices, runs of its
    rows too, are constants."""

    __slots__ = ("codes", "scales", "columns", "link")

    def __init__(self, codes, scales, columns, link=None):
        self.codes, self.scales, self.columns, self.link = codes, scales, int(columns), link

    @property
    def shape(self):
        return (*self.codes.shape[:-1], self.columns)


# routepack_matrix, routepack_mx and routepack_ids as bytes, which take less to make
# than structures of ctypes do (a call takes about 9 microseconds, 10.5 with those).
_MATRIX, _MX, _IDS = struct.Struct("Pi4xqqq").pack, struct.Struct("PPqq").pack, struct.Struct("Pi4xqqq").pack


class _ExpertCall(_Call):
    __slots__ = ()

    def on_device(self, x):
        """Whether x is a tensor on the call's GPU (the first one decides)."""
        if type(x) is not self.torch.Tensor or not x.is_cuda:
            return False
        if self.device is None:
            self.device = x.device
            return True
        return x.device == self.device

    def mx(self, name, q, dims):
        """An Mx of `dims` axes: (its codes' shape, its rows for the library)."""
        torch = self.torch
        if not isinstance(q, Mx):
            raise TypeError(f"{self.fn}: {name} must be an Mx, got {type(q).__name__}")
        codes, scales, cols = q.codes, q.scales, q.columns
        n = (cols + 127) // 128
        if self.on_device(codes) and self.on_device(scales) and codes.dtype is torch.uint8 and scales.dtype is torch.uint8:
            shape, s = codes.shape, scales.shape
            if (len(shape) == len(s) == dims and shape[-1] == 64 * n and s[-1] == 4 * n and cols >= 0 and shape[0] == s[0]
                    and (dims == 2 or shape[1] == s[1]) and codes.is_contiguous() and scales.is_contiguous()):
                return shape, _MX(codes.data_ptr(), scales.data_ptr(), shape[0] if dims == 2 else shape[0] * shape[1], cols)
        # what is wrong with it (or a subclass of Tensor)
        codes = self.tensor(f"{name}.codes", codes, (torch.uint8,))
        scales = self.tensor(f"{name}.scales", scales, (torch.uint8,))
        shape = codes.shape
        if len(shape) != dims or cols < 0 or shape[-1] != 64 * n or scales.shape != (*shape[:-1], 4 * n):
            raise ValueError(f"{self.fn}: {name} has codes {tuple(shape)} and scales {tuple(scales.shape)} for "
                             f"{cols} columns, expected {dims} axes, the last {64 * n} and {4 * n}")
        if not codes.is_contiguous() or not scales.is_contiguous():
            raise ValueError(f"{self.fn}: {name} must be contiguous")
        return shape, _MX(codes.data_ptr(), scales.data_ptr(), shape[0] if dims == 2 else shape[0] * shape[1], cols)

    def matrix(self, name, x, types):
        """[rows][columns] with adjacent columns."""
        self.tensor(name, x, types)
        shape, stride = x.shape, x.stride()
        if len(shape) != 2:
            raise ValueError(f"{self.fn}: {name} has shape {tuple(shape)}, expected [rows][columns]")
        if shape[1] > 1 and stride[1] != 1 and shape[0] > 0:
            raise ValueError(f"{self.fn}: the columns of {name} must be adjacent in memory")
        return shape, _MATRIX(x.data_ptr(), types[x.dtype], shape[0], shape[1], stride[0])

    def out(self, rows, cols, dtype, types):
        """A new matrix."""
        x = self.torch.empty((rows, cols), dtype=dtype, device=self.device)
        return x, _MATRIX(x.data_ptr(), types[dtype], rows, cols, cols)

    def offsets(self, order, n_slots):
        off = order.offsets if isinstance(order, Order) else order
        if self.on_device(off) and off.dtype is self.torch.int64 and off.shape == (n_slots + 1,) and off.is_contiguous():
            return off.data_ptr()
        return self.dense("offsets", off, (self.torch.int64,), (n_slots + 1,)).data_ptr()

    def places(self, order):
        if not isinstance(order, Order):
            raise TypeError(f"{self.fn}: order must be an Order, got {type(order).__name__}")
        p = self.tensor("order.places", order.places, (self.torch.int32,))
        shape, stride = p.shape, p.stride()
        if len(shape) != 2 or shape[1] < 1 or (shape[1] > 1 and stride[1] != 1 and shape[0] > 0):
            raise ValueError(f"{self.fn}: order.places has shape {tuple(shape)}, expected [T][k], choices adjacent")
        return shape, _IDS(p.data_ptr(), 5, shape[0], stride[0], 0)

    def gates(self, gates, shape):
        if gates is None:
            return None, 0
        g = self.tensor("gates", gates, (self.torch.float32,), shape)
        stride = g.stride()
        if shape[1] > 1 and stride[1] != 1 and shape[0] > 0:
            raise ValueError(f"{self.fn}: a token's gates must be adjacent in memory")
        return g.data_ptr(), stride[0]


def order_tokens(prob: Problem, ids, *, slots=None):
    """The Order of the pairs of tokens and chosen experts: by slot, and by pair
    within a slot.

    ids [T][L][k] (or [T][k] where L is 1) uint8, int16, int32 or int64, any
    strides over tokens and layers; ids outside [0, E) are no choices.  slots:
    int32 [L][E], place_experts' slot of each expert; without it the experts
    are the slots.  For ids [T][k] the order is one layer's; for [T][L][k] it
    has a layer axis (`Order.layer`)."""
    lib, torch, _, ints = _router()
    call = _Call("routepack_order_tokens", torch)
    shape, x = call.rows("ids", ids, ints, prob.n_layers, prob.top_k)
    L, E, at = prob.n_layers, prob.n_experts, call.device
    s = None if slots is None else call.dense("slots", slots, (torch.int32,), (L, E)).data_ptr()
    lead = () if len(shape) == 2 else (L,)
    rows = torch.empty((*lead, shape[0] * prob.top_k), dtype=torch.int32, device=at)
    offsets = torch.empty((*lead, E + 1), dtype=torch.int64, device=at)
    places = torch.empty(shape, dtype=torch.int32, device=at)
    size = lib.routepack_order_workspace(prob.ref, shape[0])
    # (kept until the kernels stand in the stream: only then may another thread's call have it)
    work = torch.empty(size, dtype=torch.uint8, device=at) if size > 0 else None
    call.run(lib.routepack_order_tokens, prob.ref, C.byref(x), s, rows.data_ptr(), offsets.data_ptr(),
             places.data_ptr(), None if work is None else work.data_ptr(), size)
    return Order(rows, offsets, places)


def quantize_mx(x, *, order=None):
    """x [rows][columns] (or [n][rows][columns], contiguous) fp32, bf16 or fp16,
    any stride over rows, as an Mx.  With `order` the result's rows are the
    order's pairs: row r holds the token of pair rows[r] (zeros behind the
    last).

    Where x requires a gradient, autograd records the quantization as if it were
    the identity: expert_product and dequantize_mx pass x's gradient back through
    the result, with `order` (of at most 32 choices) as the sum of a token's
    rows, which is combine_tokens'."""
    lib, torch, floats, _ = _router()
    call = _ExpertCall("routepack_quantize_mx", torch)
    call.tensor("x", x, floats)
    if x.requires_grad and torch.is_grad_enabled():
        codes, scales, link = _expert_functions()[2].apply(x, order)
        return Mx(codes, scales, x.shape[-1], link)
    lead = x.shape[:-1]
    if x.dim() == 3 and order is None and x.is_contiguous():
        x = x.view(-1, x.shape[-1]) if x.numel() else x.reshape(lead[0] * lead[1], x.shape[-1])
    shape, m = call.matrix("x", x, floats)
    rows, p, k = None, None, 1
    if order is not None:
        got, p = call.places(order)
        if got[0] != shape[0]:
            raise ValueError(f"{call.fn}: the order has {got[0]} tokens, x {shape[0]} rows")
        k, lead = got[1], (got[0] * got[1],)
        rows = call.dense("order.rows", order.rows, (torch.int32,), lead).data_ptr()
    n = (shape[1] + 127) // 128
    codes = torch.empty((*lead, 64 * n), dtype=torch.uint8, device=call.device)
    scales = torch.empty((*lead, 4 * n), dtype=torch.uint8, device=call.device)
    q = _MX(codes.data_ptr(), scales.data_ptr(), shape[0] if order is None else lead[0], shape[1])
    call.run(lib.routepack_quantize_mx, m, rows, p, k, q)
    return Mx(codes, scales, shape[1])


def dequantize_mx(q: Mx, dtype=None):
    """The values of an Mx as a tensor of its shape (bf16 unless `dtype` is
    given; exact in fp32 and bf16)."""
    lib, torch, floats, _ = _router()
    call = _ExpertCall("routepack_dequantize_mx", torch)
    dtype = torch.bfloat16 if dtype is None else dtype
    if dtype not in floats:
        raise ValueError(f"{call.fn}: dtype is {dtype}")
    if isinstance(q, Mx) and q.link is not None and torch.is_grad_enabled():
        return _expert_functions()[3].apply(q.link, q, dtype)
    shape, m = call.mx("q", q, 3 if isinstance(q, Mx) and q.codes.dim() == 3 else 2)
    cols = q.columns
    rows = shape[0] if len(shape) == 2 else shape[0] * shape[1]
    x = torch.empty((*shape[:-1], cols), dtype=dtype, device=call.device)
    call.run(lib.routepack_dequantize_mx, m, _MATRIX(x.data_ptr(), floats[dtype], rows, cols, cols))
    return x


def expert_product(x, w, order, *, dtype=None):
    """y [P][N]: each slot's rows of x times its matrix,
    y[r] = w[s] x[r] for r in [offsets[s], offsets[s + 1]), 0 in rows of no slot.

    x: Mx [P][C]; w: Mx [E][N][C]; order: an Order, or its offsets (int64
    [E + 1]).  Either may be a tensor (fp32, bf16, fp16) instead, which the call
    quantizes.  y has type `dtype`, by default x's type if that is a tensor, else
    bf16.  Where such tensors, or those that an Mx was quantized from, require a
    gradient, autograd records the product; the gradient passes the quantization
    as if it were the identity, and is expert_product_backward's: formed in y's
    type, and only then brought to the tensor's (a gradient in fp32 of fp32
    weights asks for dtype=torch.float32)."""
    lib, torch, floats, _ = _router()
    call = _ExpertCall("routepack_expert_product", torch)
    x_is, w_is = isinstance(x, torch.Tensor), isinstance(w, torch.Tensor)
    if dtype is None:
        dtype = x.dtype if x_is else torch.bfloat16
    if dtype not in floats:
        raise ValueError(f"{call.fn}: dtype is {dtype}")
    # what the gradients go to
    x_to, w_to = x if x_is else getattr(x, "link", None), w if w_is else getattr(w, "link", None)
    if x_to is not None or w_to is not None:
        if ((x_to is not None and x_to.requires_grad or w_to is not None and w_to.requires_grad)
                and torch.is_grad_enabled()):
            return _expert_functions()[0].apply(x_to, w_to, None if x_is else x, None if w_is else w, order, dtype)
        x, w = quantize_mx(x) if x_is else x, quantize_mx(w) if w_is else w
    got, xm = call.mx("x", x, 2)
    shape, wm = call.mx("w", w, 3)
    if x.columns != w.columns:
        raise ValueError(f"{call.fn}: x has {x.columns} columns, w {w.columns}")
    off = call.offsets(order, shape[0])
    y, ym = call.out(got[0], shape[1], dtype, floats)
    call.run(lib.routepack_expert_product, xm, wm, shape[0], off, ym)
    return y


def expert_product_backward(dy, x, w, order, *, need=(True, True)):
    """(dx [P][C], dw [E][N][C]), both of dy's type, of expert_product's y given
    its gradient dy [P][N] (fp32, bf16 or fp16, any stride over rows); None for
    what `need` leaves out.  x and w are the Mx of the product (x may be None
    where dw is not needed, and w where dx is not, but for its shape: then give
    (E, N, columns))."""
    lib, torch, floats, _ = _router()
    call = _ExpertCall("routepack_expert_product_backward", torch)
    got, dm = call.matrix("dy", dy, floats)
    if not any(need):
        raise ValueError(f"{call.fn}: neither gradient is needed")
    if isinstance(w, Mx):
        shape, wm = call.mx("w", w, 3)
        E, N, cols = shape[0], shape[1], w.columns
    elif need[0]:
        raise TypeError(f"{call.fn}: w must be an Mx, got {type(w).__name__}")
    else:
        E, N, cols = w
        wm = _MX(0, 0, E * N, cols)
    if isinstance(x, Mx):
        xs, xm = call.mx("x", x, 2)
        if xs[0] != got[0] or x.columns != cols:
            raise ValueError(f"{call.fn}: x has {xs[0]} rows of {x.columns}, dy {got[0]} rows, w {cols} columns")
    elif need[1]:
        raise TypeError(f"{call.fn}: x must be an Mx, got {type(x).__name__}")
    else:
        xm = _MX(0, 0, got[0], cols)
    if got[1] != N:
        raise ValueError(f"{call.fn}: dy has {got[1]} columns, w {N} rows a slot")
    off = call.offsets(order, E)
    dx = dw = dxm = dwm = None
    if need[0]:
        dx, dxm = call.out(got[0], cols, dy.dtype, floats)
    if need[1]:
        dw = torch.empty((E, N, cols), dtype=dy.dtype, device=call.device)
        dwm = _MATRIX(dw.data_ptr(), floats[dy.dtype], E * N, cols, cols)
    call.run(lib.routepack_expert_product_backward, dm, xm, wm, E, off, dxm, dwm)
    return dx, dw


def combine_tokens(y, order, gates=None):
    """out [T][C] = sum over a token's choices of gate times row: y [P][C] fp32,
    bf16 or fp16, any stride over rows; gates float32 [T][k], any stride over
    tokens (ones if None); order: one layer's Order.  Sums run in 32 bits in the
    order of the choices; out has y's type.  Where y or the gates require a
    gradient, autograd records the sum; its backward pass is combine_backward's."""
    lib, torch, floats, _ = _router()
    call = _ExpertCall("routepack_combine_tokens", torch)
    got, ym = call.matrix("y", y, floats)
    shape, p = call.places(order)
    g, stride = call.gates(gates, shape)
    if (y.requires_grad or (gates is not None and gates.requires_grad)) and torch.is_grad_enabled():
        return _expert_functions()[1].apply(y, gates, order)
    out, om = call.out(shape[0], got[1], y.dtype, floats)
    call.run(lib.routepack_combine_tokens, ym, p, shape[1], g, stride, om)
    return out


def combine_backward(dout, y, order, gates=None, *, need=(True, True)):
    """(dy [P][C] of y's type, dgates float32 [T][k]) of combine_tokens' sum given
    its gradient dout [T][C] of y's type; None for what `need` leaves out."""
    lib, torch, floats, _ = _router()
    call = _ExpertCall("routepack_combine_backward", torch)
    got, ym = call.matrix("y", y, floats)
    dshape, dm = call.matrix("dout", dout, {y.dtype: floats[y.dtype]})
    shape, p = call.places(order)
    g, stride = call.gates(gates, shape)
    if tuple(dshape) != (shape[0], got[1]):
        raise ValueError(f"{call.fn}: dout has shape {tuple(dshape)}, expected {(shape[0], got[1])}")
    if not any(need):
        raise ValueError(f"{call.fn}: neither gradient is needed")
    dy = dgates = dym = rows = None
    if need[0]:
        rows = call.dense("order.rows", order.rows, (torch.int32,), (got[0],)).data_ptr()
        dy, dym = call.out(got[0], got[1], y.dtype, floats)
    if need[1]:
        dgates = torch.empty(tuple(shape), dtype=torch.float32, device=call.device)
        if dy is None and shape[0] == 0:  # (no token: nothing to write, and no address to pass)
            return None, dgates
    call.run(lib.routepack_combine_backward, dm, ym, rows, p, shape[1], g, stride, dym,
             None if dgates is None else dgates.data_ptr())
    return dy, dgates


_EXPERT_FUNCTIONS = None


def _expert_functions():
    """(product, sum, quantization, values) as functions that autograd records."""
    global _EXPERT_FUNCTIONS
    if _EXPERT_FUNCTIONS is not None:
        return _EXPERT_FUNCTIONS
    torch = _router()[1]
    once_differentiable = torch.autograd.function.once_differentiable

    class Product(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x_to, w_to, x, w, order, dtype):
            qx, qw = quantize_mx(x_to) if x is None else x, quantize_mx(w_to) if w is None else w
            off = order.offsets if isinstance(order, Order) else order
            # (the packed matrices are kept, a quarter of the tensors in bf16)
            need = ctx.needs_input_grad
            none = qx.codes.new_empty(0)
            ctx.save_for_backward(qx.codes if need[1] else none, qx.scales if need[1] else none,
                                  qw.codes if need[0] else none, qw.scales if need[0] else none, off)
            ctx.sizes = (*qw.shape[:2], qw.columns), [None if t is None else t.dtype for t in (x_to, w_to)]
            return expert_product(qx, qw, off, dtype=dtype)

        @staticmethod
        @once_differentiable
        def backward(ctx, dy):
            xc, xs, wc, ws, off = ctx.saved_tensors
            sizes, types = ctx.sizes
            need = tuple(ctx.needs_input_grad[:2])
            if dy.dim() == 2 and dy.stride(1) != 1:
                dy = dy.contiguous()
            dx, dw = expert_product_backward(dy, Mx(xc, xs, sizes[2]) if need[1] else None,
                                             Mx(wc, ws, sizes[2]) if need[0] else sizes, off, need=need)
            return (None if dx is None else dx.to(types[0]), None if dw is None else dw.to(types[1])) + (None,) * 4

    class Sum(torch.autograd.Function):
        @staticmethod
        def forward(ctx, y, gates, order):
            ctx.save_for_backward(y, gates, order.rows, order.places)
            return combine_tokens(y, order, gates)

        @staticmethod
        @once_differentiable
        def backward(ctx, dout):
            y, gates, rows, places = ctx.saved_tensors
            if dout.stride(1) != 1:
                dout = dout.contiguous()
            dy, dgates = combine_backward(dout, y, Order(rows, None, places), gates,
                                          need=tuple(ctx.needs_input_grad[:2]))
            return dy, dgates, None

    class Quantize(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, order):
            q = quantize_mx(x, order=order)
            if order is not None and order.places.shape[1] > 32:  # (combine_tokens' limit)
                raise ValueError(f"routepack_quantize_mx: x requires a gradient, and the order has {order.places.shape[1]} "
                                 "choices, more than 32")
            ctx.gathered = order is not None
            if ctx.gathered:
                ctx.save_for_backward(order.places)
            ctx.mark_non_differentiable(q.codes, q.scales)
            ctx.set_materialize_grads(False)
            # (one element for all: only its shape, type and place in the graph count)
            link = torch.empty_strided(q.shape, (0,) * len(q.shape), dtype=x.dtype, device=x.device)
            return q.codes, q.scales, link

        @staticmethod
        @once_differentiable
        def backward(ctx, _, __, dlink):
            if dlink is None or not ctx.gathered:
                return dlink, None
            (places,) = ctx.saved_tensors
            if dlink.stride(1) != 1:
                dlink = dlink.contiguous()
            return combine_tokens(dlink, Order(None, None, places)), None

    class Values(torch.autograd.Function):
        @staticmethod
        def forward(ctx, link, q, dtype):
            ctx.type = link.dtype
            return dequantize_mx(q, dtype)

        @staticmethod
        @once_differentiable
        def backward(ctx, dx):
            return dx.to(ctx.type), None, None

    _EXPERT_FUNCTIONS = Product, Sum, Quantize, Values
    return _EXPERT_FUNCTIONS
