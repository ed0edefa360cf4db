"""UltraEP per-microbatch balancing path for MI355X (gfx950), and the operators
of the MoE layer around it.

Thin ctypes binding of ``libultraep.so`` (C ABI in ``include/ultraep.h``).
Every function has the name of the C entry point it calls and only marshals
arguments: torch tensors supply device memory, torch's current HIP stream is
used unless another one is given, and every step runs in the library's HIP
kernels.  Before a call it checks that every tensor is large enough for the
shapes given, so a kernel never runs past a caller's buffer.  A call whose
arguments pass the checks goes through ``_native.so`` (``csrc/binding.cpp``),
which makes them in C++; one that it does not take (None is returned) is
checked, and refused or made, by the ctypes code below, and so is every call
where ``_native.so`` is not built for this torch.  A missing library raises
immediately; there is no fallback for the kernels.

Reference: "UltraEP: Unleash MoE Training and Inference on Rack-Scale Nodes
with Near-Optimal Load Balancing", arXiv 2606.04101 (Algorithm 1, Sec. 5-6).
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
# the in-tree build; ULTRAEP_LIB names another build of the same sources
# (for example a kernel variant under comparison) without replacing it
LIB_PATH = os.environ.get("ULTRAEP_LIB") or os.path.join(_HERE, "libultraep.so")

ULTRAEP_OK = 0
ULTRAEP_EINVAL = -1
ULTRAEP_ENOSPC = -2
ULTRAEP_EDEVICE = -3
ULTRAEP_EDATA = -4


class UltraEPError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {ultraep_strerror(code)} ({code})")


class Group(ctypes.Structure):
    """ultraep_group: R ranks, E experts, n_slot redundant slots per rank,
    quota floor u_min, balancing target beta_num / beta_den."""
    _fields_ = [("R", ctypes.c_int32), ("E", ctypes.c_int32),
                ("n_slot", ctypes.c_int32), ("u_min", ctypes.c_int64),
                ("beta_num", ctypes.c_int32), ("beta_den", ctypes.c_int32)]

    def __init__(self, R, E, n_slot, u_min, beta_num=101, beta_den=100):
        super().__init__(R, E, n_slot, u_min, beta_num, beta_den)

    @property
    def n_main(self):
        return self.E // self.R

    @property
    def S(self):
        return self.n_main + self.n_slot

    @property
    def ncol(self):
        return self.E + self.R * self.n_slot


class PlanBuf(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("slot_expert", "quota", "host_ptr", "host_rank", "host_pslot",
                 "reroute", "stats")]


ULTRAEP_F32, ULTRAEP_BF16 = 0, 1
ULTRAEP_SOFTMAX, ULTRAEP_SIGMOID = 0, 1


class Router(ctypes.Structure):
    """ultraep_router: E experts, k of them a token, the score function
    (ULTRAEP_SOFTMAX or ULTRAEP_SIGMOID), gates renormalised over a token's
    experts and scaled, the best top_group of n_group groups (0: all eligible),
    seq_len tokens a sequence in the statistics (0: all are one)."""
    _fields_ = [("E", ctypes.c_int32), ("k", ctypes.c_int32), ("score", ctypes.c_int32),
                ("renorm", ctypes.c_int32), ("n_group", ctypes.c_int32),
                ("top_group", ctypes.c_int32), ("scale", ctypes.c_float),
                ("seq_len", ctypes.c_int64)]

    def __init__(self, E, k, score=ULTRAEP_SOFTMAX, renorm=True, n_group=0, top_group=0, scale=1.0,
                 seq_len=0):
        super().__init__(E, k, score, int(renorm), n_group, top_group, scale, seq_len)

    def n_seg(self, T):
        """Sequences of T tokens."""
        return -(-T // self.seq_len) if self.seq_len > 0 and T > 0 else 1


PLAN_FIELDS = ("slot_expert", "quota", "host_ptr", "host_rank", "host_pslot",
               "reroute", "stats")

_lib = None
_native = None
_P = ctypes.c_void_p


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is not built; run __graft_entry__.build() first")
        L = ctypes.CDLL(LIB_PATH)
        i32, i64, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        gp, pp = ctypes.POINTER(Group), ctypes.POINTER(PlanBuf)
        L.ultraep_plan_sizes.argtypes = [gp, ctypes.POINTER(sz)]
        L.ultraep_count.argtypes = [_P, i64, i32, i32, i32, _P, _P, _P]
        L.ultraep_plan.argtypes = [_P, gp, pp, _P, sz, _P]
        L.ultraep_plan_noalloc.argtypes = [_P, gp, pp, _P]
        L.ultraep_plan_replicate.argtypes = [_P, gp, pp, _P, sz, _P]
        L.ultraep_plan_reroute.argtypes = [_P, gp, pp, _P]
        L.ultraep_plan_ws_bytes.argtypes = [gp]
        L.ultraep_plan_ws_bytes.restype = sz
        L.ultraep_dispatch_ws_bytes.argtypes = [i64, i32, gp]
        L.ultraep_dispatch_ws_bytes.restype = sz
        L.ultraep_dispatch.argtypes = [_P, _P, i64, i32, i32, i32, gp, pp, _P,
                                       _P, _P, _P, sz, _P, _P]
        L.ultraep_dispatch_layout.argtypes = [_P, i64, i32, i32, gp, pp, _P, _P,
                                              _P, sz, _P, _P]
        L.ultraep_dispatch_scatter.argtypes = [_P, i64, i32, i32, _P, _P, _P, _P]
        L.ultraep_pack_replicas.argtypes = [_P, i64, i32, gp, pp, _P, i64, _P,
                                            _P, _P]
        L.ultraep_reroute_and_pack.argtypes = [_P, gp, pp, _P, i64, i32, _P, i64, _P,
                                               _P, _P]
        L.ultraep_relay_plan.argtypes = [gp, pp, i32, _P, _P, _P, _P, _P]
        L.ultraep_pack_relay.argtypes = [_P, _P, i64, i32, gp, pp, _P, _P, i64, _P,
                                         _P, _P]
        L.ultraep_combine.argtypes = [_P, i64, _P, _P, i64, i32, i32, _P, _P, _P]
        L.ultraep_grad_reduce.argtypes = [_P, _P, i64, i32, gp, pp, i64, _P, _P]
        f32, rp = ctypes.c_float, ctypes.POINTER(Router)
        L.ultraep_route_ws_bytes.argtypes = [i64, rp]
        L.ultraep_route_ws_bytes.restype = sz
        L.ultraep_route.argtypes = [_P, i32, i64, i64, rp, _P, _P, _P, _P, _P, _P, _P, _P, sz,
                                    _P, _P]
        L.ultraep_balance_loss.argtypes = [_P, _P, _P, _P, i64, rp, f32, _P, _P, _P]
        L.ultraep_route_grad.argtypes = [_P, i32, i64, i64, rp, _P, _P, _P, _P, _P, _P, _P, _P]
        L.ultraep_combine_grad.argtypes = [_P, _P, i64, _P, _P, i64, i32, i32, _P, _P, _P, _P, _P]
        L.ultraep_quant_rows.argtypes = [_P, i32, i64, i64, i64, _P, i64, _P, _P]
        L.ultraep_expert_matmul.argtypes = [_P, _P, i64, _P, _P, i32, i32, i32, _P, _P, i32, i32,
                                            _P, i32, _P, _P]
        L.ultraep_strerror.argtypes = [ctypes.c_int]
        L.ultraep_strerror.restype = ctypes.c_char_p
        for f in ("ultraep_plan_sizes", "ultraep_count", "ultraep_plan",
                  "ultraep_plan_noalloc", "ultraep_plan_replicate", "ultraep_plan_reroute",
                  "ultraep_dispatch", "ultraep_dispatch_layout",
                  "ultraep_dispatch_scatter", "ultraep_pack_replicas",
                  "ultraep_reroute_and_pack", "ultraep_relay_plan",
                  "ultraep_pack_relay", "ultraep_combine", "ultraep_grad_reduce",
                  "ultraep_route", "ultraep_balance_loss", "ultraep_route_grad",
                  "ultraep_combine_grad", "ultraep_quant_rows", "ultraep_expert_matmul"):
            getattr(L, f).restype = ctypes.c_int
        _lib = L
    return _lib


class _Declines:
    """In place of the native half where there is none: it takes no call, so
    every call goes through the ctypes code."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_native():
    """The native half of the binding, bound to the library's entry points; a
    stand-in that takes no call, and a warning, where it is not built or was
    built for another torch (the calls then cost more host time, 5-8 us each)."""
    global _native
    L = lib()
    try:
        import importlib

        import torch  # the module links against torch's libraries
        m = importlib.import_module("._native", __name__)
        if m.torch_version != str(torch.__version__):
            raise ImportError(f"it was built for torch {m.torch_version}")
    except (ImportError, AttributeError) as e:
        import warnings
        warnings.warn(f"{__name__}: calls go through ctypes, the native half of the binding "
                      f"does not load: {e}", RuntimeWarning, stacklevel=3)
        m = _Declines()
    else:
        m.bind({f"ultraep_{n}": ctypes.cast(getattr(L, f"ultraep_{n}"), _P).value
                for n in ("count", "plan", "plan_noalloc", "plan_replicate", "plan_reroute",
                          "dispatch", "dispatch_layout", "dispatch_scatter", "pack_replicas",
                          "reroute_and_pack", "relay_plan", "pack_relay", "combine",
                          "grad_reduce", "route", "balance_loss", "route_grad",
                          "combine_grad", "quant_rows", "expert_matmul")},
               Group, Plan, PlanBuf, Router)
    _native = m
    return m


def ultraep_strerror(code: int) -> str:
    return lib().ultraep_strerror(int(code)).decode()


def _check(rc, where):
    if rc != ULTRAEP_OK:
        raise UltraEPError(rc, where)
    return rc


def _ptr(t):
    """Device address of a torch tensor (None for None / empty tensors)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return t.data_ptr() if t.numel() else None


def _need(t, n, esize, name):
    """Raises unless t holds at least n elements of esize bytes, so that no
    kernel reads or writes past a caller's tensor (n <= 0 needs nothing)."""
    if n <= 0:
        return
    if t is None:
        raise ValueError(f"{name}: a device tensor of {n} elements is needed")
    if t.element_size() != esize:
        raise ValueError(f"{name}: expected {esize}-byte elements, got {t.dtype}")
    if t.numel() < n:
        raise ValueError(f"{name}: needs {n} elements, has {t.numel()}")


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream
    import torch
    return torch.cuda.current_stream().cuda_stream


def ultraep_plan_sizes(g: Group):
    out = (ctypes.c_size_t * 7)()
    _check(lib().ultraep_plan_sizes(ctypes.byref(g), out), "ultraep_plan_sizes")
    return tuple(int(v) for v in out)


class Plan:
    """Device buffers of one plan (torch tensors), their C descriptor, and the
    planner's device workspace."""

    def __init__(self, g: Group, device="cuda"):
        import torch
        n = ultraep_plan_sizes(g)
        dt = [torch.int32] * 6 + [torch.int64]
        for name, cnt, d in zip(PLAN_FIELDS, n, dt):
            setattr(self, name, torch.empty(cnt, dtype=d, device=device))
        self.g = g
        self.c = PlanBuf(*[_ptr(getattr(self, f)) for f in PLAN_FIELDS])
        self.ws = torch.empty(ultraep_plan_ws_bytes(g), dtype=torch.uint8,
                              device=device)


def ultraep_count(topk, T, k, E, n_groups, counts, status, stream=None):
    rc = (_native or _load_native()).count(topk, T, k, E, n_groups, counts, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_count")
    _need(topk, n_groups * T * k, 4, "topk")
    _need(counts, n_groups * E, 4, "counts")
    _need(status, 1, 4, "status")
    return _check(lib().ultraep_count(_ptr(topk), T, k, E, n_groups,
                                      _ptr(counts), _ptr(status),
                                      _stream(stream)), "ultraep_count")


def ultraep_plan_ws_bytes(g: Group) -> int:
    return int(lib().ultraep_plan_ws_bytes(ctypes.byref(g)))


def ultraep_plan(load, g: Group, plan: Plan, ws=None, stream=None):
    """ws: device workspace (defaults to the one the Plan object holds)."""
    rc = (_native or _load_native()).plan(load, g, plan, ws, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_plan")
    ws = plan.ws if ws is None else ws
    _need(load, g.R * g.E, 4, "load")
    return _check(lib().ultraep_plan(_ptr(load), ctypes.byref(g),
                                     ctypes.byref(plan.c), _ptr(ws),
                                     ws.numel() * ws.element_size(),
                                     _stream(stream)), "ultraep_plan")


def ultraep_plan_noalloc(load, g: Group, plan: Plan, stream=None):
    """ultraep_plan with the library's fixed per-device workspace (plan.ws is
    not used); calls on one device must not overlap in time."""
    rc = (_native or _load_native()).plan_noalloc(load, g, plan, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_plan_noalloc")
    _need(load, g.R * g.E, 4, "load")
    return _check(lib().ultraep_plan_noalloc(_ptr(load), ctypes.byref(g),
                                             ctypes.byref(plan.c), _stream(stream)),
                  "ultraep_plan_noalloc")


def ultraep_plan_replicate(load, g: Group, plan: Plan, ws=None, stream=None):
    rc = (_native or _load_native()).plan_replicate(load, g, plan, ws, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_plan_replicate")
    ws = plan.ws if ws is None else ws
    _need(load, g.R * g.E, 4, "load")
    return _check(lib().ultraep_plan_replicate(
        _ptr(load), ctypes.byref(g), ctypes.byref(plan.c), _ptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)), "ultraep_plan_replicate")


def ultraep_plan_reroute(load, g: Group, plan: Plan, stream=None):
    rc = (_native or _load_native()).plan_reroute(load, g, plan, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_plan_reroute")
    _need(load, g.R * g.E, 4, "load")
    return _check(lib().ultraep_plan_reroute(
        _ptr(load), ctypes.byref(g), ctypes.byref(plan.c), _stream(stream)),
        "ultraep_plan_reroute")


def ultraep_dispatch_ws_bytes(T, k, g: Group) -> int:
    return int(lib().ultraep_dispatch_ws_bytes(T, k, ctypes.byref(g)))


def _layout_need(topk, T, k, g, row_of_slot, block_off, status):
    _need(topk, T * k, 4, "topk")
    _need(row_of_slot, T * k, 4, "row_of_slot")
    _need(block_off, g.R * g.S + 1, 8, "block_off")
    _need(status, 1, 4, "status")


def ultraep_dispatch(x, topk, T, k, H, rank, g: Group, plan: Plan, send,
                     row_of_slot, block_off, ws, status, stream=None):
    rc = (_native or _load_native()).dispatch(x, topk, T, k, H, rank, g, plan, send, row_of_slot,
                                             block_off, ws, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_dispatch")
    _need(x, T * H, 2, "x")
    _need(send, T * k * H, 2, "send")
    _layout_need(topk, T, k, g, row_of_slot, block_off, status)
    return _check(lib().ultraep_dispatch(
        _ptr(x), _ptr(topk), T, k, H, rank, ctypes.byref(g),
        ctypes.byref(plan.c), _ptr(send), _ptr(row_of_slot), _ptr(block_off),
        _ptr(ws), ws.numel() * ws.element_size(), _ptr(status),
        _stream(stream)), "ultraep_dispatch")


def ultraep_dispatch_layout(topk, T, k, rank, g: Group, plan: Plan,
                            row_of_slot, block_off, ws, status, stream=None):
    rc = (_native or _load_native()).dispatch_layout(topk, T, k, rank, g, plan, row_of_slot,
                                                    block_off, ws, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_dispatch_layout")
    _layout_need(topk, T, k, g, row_of_slot, block_off, status)
    return _check(lib().ultraep_dispatch_layout(
        _ptr(topk), T, k, rank, ctypes.byref(g), ctypes.byref(plan.c),
        _ptr(row_of_slot), _ptr(block_off), _ptr(ws),
        ws.numel() * ws.element_size(), _ptr(status), _stream(stream)),
        "ultraep_dispatch_layout")


def ultraep_dispatch_scatter(x, T, k, H, row_of_slot, n_routed, send,
                             stream=None):
    """n_routed: a one-element int64 device tensor (e.g. block_off[-1:])."""
    rc = (_native or _load_native()).dispatch_scatter(x, T, k, H, row_of_slot, n_routed, send,
                                                     stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_dispatch_scatter")
    _need(x, T * H, 2, "x")
    _need(row_of_slot, T * k, 4, "row_of_slot")
    _need(n_routed, 1 if T > 0 else 0, 8, "n_routed")
    _need(send, T * k * H, 2, "send")
    return _check(lib().ultraep_dispatch_scatter(
        _ptr(x), T, k, H, _ptr(row_of_slot), _ptr(n_routed), _ptr(send),
        _stream(stream)), "ultraep_dispatch_scatter")


def _pack_need(w_main, W, g, staging, cap, dest_off, status):
    _need(w_main, g.n_main * W, 2, "w_main")
    _need(staging, cap * W, 2, "staging")
    _need(dest_off, g.R + 1, 8, "dest_off")
    _need(status, 1, 4, "status")


def ultraep_pack_replicas(w_main, W, rank, g: Group, plan: Plan, staging, cap,
                          dest_off, status, stream=None):
    rc = (_native or _load_native()).pack_replicas(w_main, W, rank, g, plan, staging, cap,
                                                  dest_off, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_pack_replicas")
    _pack_need(w_main, W, g, staging, cap, dest_off, status)
    return _check(lib().ultraep_pack_replicas(
        _ptr(w_main), W, rank, ctypes.byref(g), ctypes.byref(plan.c),
        _ptr(staging), cap, _ptr(dest_off), _ptr(status), _stream(stream)),
        "ultraep_pack_replicas")


def ultraep_reroute_and_pack(load, g: Group, plan: Plan, w_main, W, rank, staging,
                             cap, dest_off, status, stream=None):
    rc = (_native or _load_native()).reroute_and_pack(load, g, plan, w_main, W, rank, staging,
                                                     cap, dest_off, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_reroute_and_pack")
    _need(load, g.R * g.E, 4, "load")
    _pack_need(w_main, W, g, staging, cap, dest_off, status)
    return _check(lib().ultraep_reroute_and_pack(
        _ptr(load), ctypes.byref(g), ctypes.byref(plan.c), _ptr(w_main), W, rank,
        _ptr(staging), cap, _ptr(dest_off), _ptr(status), _stream(stream)),
        "ultraep_reroute_and_pack")


def ultraep_relay_plan(g: Group, plan: Plan, threshold, slot_src, send_vol,
                       relay_stats, status, stream=None):
    rc = (_native or _load_native()).relay_plan(g, plan, threshold, slot_src, send_vol,
                                               relay_stats, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_relay_plan")
    _need(slot_src, g.R * g.n_slot, 4, "slot_src")
    _need(send_vol, g.R, 4, "send_vol")
    _need(relay_stats, 4, 8, "relay_stats")
    _need(status, 1, 4, "status")
    return _check(lib().ultraep_relay_plan(
        ctypes.byref(g), ctypes.byref(plan.c), threshold, _ptr(slot_src),
        _ptr(send_vol), _ptr(relay_stats), _ptr(status), _stream(stream)),
        "ultraep_relay_plan")


def ultraep_pack_relay(w_main, relay_src, W, rank, g: Group, plan: Plan, slot_src,
                       staging, cap, dest_off, status, stream=None):
    rc = (_native or _load_native()).pack_relay(w_main, relay_src, W, rank, g, plan, slot_src,
                                               staging, cap, dest_off, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_pack_relay")
    _pack_need(w_main, W, g, staging, cap, dest_off, status)
    _need(relay_src, g.n_slot * W, 2, "relay_src")
    _need(slot_src, g.R * g.n_slot, 4, "slot_src")
    return _check(lib().ultraep_pack_relay(
        _ptr(w_main), _ptr(relay_src), W, rank, ctypes.byref(g), ctypes.byref(plan.c),
        _ptr(slot_src), _ptr(staging), cap, _ptr(dest_off), _ptr(status),
        _stream(stream)), "ultraep_pack_relay")


def ultraep_combine(y, n_rows, gate, row_of_slot, T, k, H, out, status, stream=None):
    rc = (_native or _load_native()).combine(y, n_rows, gate, row_of_slot, T, k, H, out, status,
                                            stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_combine")
    _need(y, n_rows * H, 2, "y")
    _need(gate, T * k, 4, "gate")
    _need(row_of_slot, T * k, 4, "row_of_slot")
    _need(out, T * H, 2, "out")
    _need(status, 1, 4, "status")
    return _check(lib().ultraep_combine(
        _ptr(y), n_rows, _ptr(gate), _ptr(row_of_slot), T, k, H, _ptr(out), _ptr(status),
        _stream(stream)), "ultraep_combine")


def ultraep_grad_reduce(main_grad, rgrad, W, rank, g: Group, plan: Plan, cap, status,
                        stream=None):
    rc = (_native or _load_native()).grad_reduce(main_grad, rgrad, W, rank, g, plan, cap, status,
                                                stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_grad_reduce")
    _need(main_grad, g.n_main * W, 4, "main_grad")
    _need(rgrad, cap * W, 4, "rgrad")
    _need(status, 1, 4, "status")
    return _check(lib().ultraep_grad_reduce(
        _ptr(main_grad), _ptr(rgrad), W, rank, ctypes.byref(g), ctypes.byref(plan.c), cap,
        _ptr(status), _stream(stream)), "ultraep_grad_reduce")


def _row_type(t, name):
    """ULTRAEP_F32 or ULTRAEP_BF16 by t's element type; bf16 may come as raw
    16-bit integers."""
    dt = str(t.dtype) if t is not None else None
    if dt == "torch.float32":
        return ULTRAEP_F32
    if dt in ("torch.bfloat16", "torch.int16", "torch.uint16"):
        return ULTRAEP_BF16
    raise ValueError(f"{name}: expected float32 or bfloat16 elements, got {dt}")


def _need_rows(t, rows, n, ld, type_, name):
    """Raises unless t holds rows of n elements, ld apart, of the row type."""
    if rows > 0:
        if _row_type(t, name) != type_:
            raise ValueError(f"{name}: expected elements of the other rows' type, got {t.dtype}")
        _need(t, (rows - 1) * ld + n, 4 if type_ == ULTRAEP_F32 else 2, name)


def ultraep_route_ws_bytes(T, r: Router) -> int:
    return int(lib().ultraep_route_ws_bytes(T, ctypes.byref(r)))


def ultraep_route(logits, T, ld, r: Router, bias, mask, topk, gate, counts, prob_sum, tokens, ws,
                  status, stream=None):
    """bias, mask, and counts, prob_sum, tokens, ws together, may be None."""
    rc = (_native or _load_native()).route(logits, T, ld, r, bias, mask, topk, gate, counts,
                                          prob_sum, tokens, ws, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_route")
    type_ = _row_type(logits, "logits") if T > 0 else ULTRAEP_F32
    n_seg = r.n_seg(T)
    _need_rows(logits, T, r.E, ld, type_, "logits")
    _need(bias, r.E if bias is not None else 0, 4, "bias")
    _need(mask, T if mask is not None else 0, 1, "mask")
    _need(topk, T * r.k, 4, "topk")
    _need(gate, T * r.k, 4, "gate")
    _need(counts, n_seg * r.E if counts is not None else 0, 4, "counts")
    _need(prob_sum, n_seg * r.E if prob_sum is not None else 0, 4, "prob_sum")
    _need(tokens, n_seg if tokens is not None else 0, 4, "tokens")
    _need(status, 1, 4, "status")
    return _check(lib().ultraep_route(
        _ptr(logits), type_, T, ld, ctypes.byref(r), _ptr(bias), _ptr(mask), _ptr(topk), _ptr(gate),
        _ptr(counts), _ptr(prob_sum), _ptr(tokens), _ptr(ws),
        ws.numel() * ws.element_size() if ws is not None else 0, _ptr(status), _stream(stream)),
        "ultraep_route")


def ultraep_balance_loss(counts, load_tokens, prob_sum, tokens, n_seg, r: Router, alpha, loss, coef,
                         stream=None):
    rc = (_native or _load_native()).balance_loss(counts, load_tokens, prob_sum, tokens, n_seg, r,
                                                 alpha, loss, coef, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_balance_loss")
    _need(counts, n_seg * r.E, 4, "counts")
    _need(load_tokens, n_seg, 4, "load_tokens")
    _need(prob_sum, n_seg * r.E, 4, "prob_sum")
    _need(tokens, n_seg, 4, "tokens")
    _need(loss, 1, 4, "loss")
    _need(coef, n_seg * r.E, 4, "coef")
    return _check(lib().ultraep_balance_loss(
        _ptr(counts), _ptr(load_tokens), _ptr(prob_sum), _ptr(tokens), n_seg, ctypes.byref(r), alpha,
        _ptr(loss), _ptr(coef), _stream(stream)), "ultraep_balance_loss")


def ultraep_route_grad(logits, T, ld, r: Router, mask, topk, dgate, coef, dloss, dlogits, status,
                       stream=None):
    """mask, dgate, coef and dloss may be None."""
    rc = (_native or _load_native()).route_grad(logits, T, ld, r, mask, topk, dgate, coef, dloss,
                                               dlogits, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_route_grad")
    type_ = _row_type(logits, "logits") if T > 0 else ULTRAEP_F32
    _need_rows(logits, T, r.E, ld, type_, "logits")
    _need_rows(dlogits, T, r.E, ld, type_, "dlogits")
    _need(mask, T if mask is not None else 0, 1, "mask")
    _need(topk, T * r.k, 4, "topk")
    _need(dgate, T * r.k if dgate is not None else 0, 4, "dgate")
    _need(coef, r.n_seg(T) * r.E if coef is not None else 0, 4, "coef")
    _need(dloss, 1 if dloss is not None else 0, 4, "dloss")
    _need(status, 1, 4, "status")
    return _check(lib().ultraep_route_grad(
        _ptr(logits), type_, T, ld, ctypes.byref(r), _ptr(mask), _ptr(topk), _ptr(dgate), _ptr(coef),
        _ptr(dloss), _ptr(dlogits), _ptr(status), _stream(stream)), "ultraep_route_grad")


def ultraep_combine_grad(dout, y, n_rows, gate, row_of_slot, T, k, H, n_routed, dy, dgate, status,
                         stream=None):
    """n_routed: a one-element int64 device tensor (e.g. block_off[-1:])."""
    rc = (_native or _load_native()).combine_grad(dout, y, n_rows, gate, row_of_slot, T, k, H,
                                                 n_routed, dy, dgate, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_combine_grad")
    _need(dout, T * H, 2, "dout")
    _need(y, n_rows * H, 2, "y")
    _need(gate, T * k, 4, "gate")
    _need(row_of_slot, T * k, 4, "row_of_slot")
    _need(n_routed, 1, 8, "n_routed")
    _need(dy, n_rows * H, 2, "dy")
    _need(dgate, T * k, 4, "dgate")
    _need(status, 1, 4, "status")
    return _check(lib().ultraep_combine_grad(
        _ptr(dout), _ptr(y), n_rows, _ptr(gate), _ptr(row_of_slot), T, k, H, _ptr(n_routed),
        _ptr(dy), _ptr(dgate), _ptr(status), _stream(stream)), "ultraep_combine_grad")


def ultraep_quant_rows(x, rows, K, ld, q, ldq, scale, stream=None):
    rc = (_native or _load_native()).quant_rows(x, rows, K, ld, q, ldq, scale, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_quant_rows")
    type_ = _row_type(x, "x") if rows > 0 else ULTRAEP_BF16
    _need_rows(x, rows, K, ld, type_, "x")
    _need(q, rows * ldq, 1, "q")
    _need(scale, rows, 4, "scale")
    return _check(lib().ultraep_quant_rows(_ptr(x), type_, rows, K, ld, _ptr(q), ldq, _ptr(scale),
                                           _stream(stream)), "ultraep_quant_rows")


def ultraep_expert_matmul(xq, x_scale, M, wq, w_scale, n_w, N, K, block_off, block_w, n_block, act,
                          y, status, stream=None):
    """block_w may be None (block g takes weight g); y is float32 or bfloat16."""
    rc = (_native or _load_native()).expert_matmul(xq, x_scale, M, wq, w_scale, n_w, N, K, block_off,
                                                  block_w, n_block, act, y, status, stream)
    if rc is not None:
        return rc if rc == ULTRAEP_OK else _check(rc, "ultraep_expert_matmul")
    type_ = _row_type(y, "y") if M > 0 else ULTRAEP_BF16
    _need(xq, M * K, 1, "xq")
    _need(x_scale, M, 4, "x_scale")
    _need(wq, n_w * N * K, 1, "wq")
    _need(w_scale, n_w * N, 4, "w_scale")
    _need(block_off, n_block + 1, 8, "block_off")
    _need(block_w, n_block if block_w is not None else 0, 4, "block_w")
    _need(y, M * (N // 2 if act else N), 4 if type_ == ULTRAEP_F32 else 2, "y")
    _need(status, 1, 4, "status")
    return _check(lib().ultraep_expert_matmul(
        _ptr(xq), _ptr(x_scale), M, _ptr(wq), _ptr(w_scale), n_w, N, K, _ptr(block_off),
        _ptr(block_w), n_block, int(act), _ptr(y), type_, _ptr(status), _stream(stream)),
        "ultraep_expert_matmul")


def build():
    """Compile libultraep.so for gfx950 in-tree."""
    from . import _build
    global _lib, _native
    _lib = _native = None
    return _build.build()
