"""Python binding of libkvevict.so (include/kv_evict.h): argument marshalling only.

Every step runs in the library's CUDA kernels; tensors are torch tensors used as
device buffers and passed by pointer. Loading fails loudly when the library has
not been built (``python -c "import __graft_entry__ as g; g.build()"``).
"""

from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libkvevict.so")

KVE_OK, KVE_EINVAL, KVE_ECUDA, KVE_ETIMEOUT, KVE_ENOMEM, KVE_EPAGES = range(6)

# Names declared in include/kv_evict.h.
EXPORTS = ("kv_evict_plan", "kv_evict_plan_layered", "kv_evict_plan_ex", "kv_evict_plan_destroy",
           "kv_evict_plan_set_debug", "kv_evict_plan_set_kv_strides",
           "kv_evict_score", "kv_evict_score_lse", "kv_evict_score_attn", "kv_evict_score_attn_workspace",
           "kv_evict_select", "kv_evict_select_noalloc", "kv_evict_select_profiles",
           "kv_evict_select_profiles_workspace", "kv_evict_gather", "kv_evict_select_gather",
           "kv_evict_status", "kv_evict_profile", "kv_evict_budget_pyramid", "kv_evict_strerror",
           "kv_evict_cache_create", "kv_evict_cache_destroy", "kv_evict_cache_reset", "kv_evict_cache_pages",
           "kv_evict_cache_gather", "kv_evict_cache_store", "kv_evict_cache_attend", "kv_evict_cache_status",
           "kv_evict_cache_append", "kv_evict_cache4_create", "kv_evict_rotary_frequencies", "kv_evict_rotary_create",
           "kv_evict_rotary_destroy", "kv_evict_rotary_apply")


class KvEvictError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {_lib().kv_evict_strerror(status).decode()} (status {status})")


class Config(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("window", ctypes.c_int32), ("budget", ctypes.c_int32),
                ("pool_kernel", ctypes.c_int32), ("candidate_factor", ctypes.c_int32),
                ("norm_eps", ctypes.c_float)]


class CacheConfig(ctypes.Structure):
    _fields_ = [("num_layers", ctypes.c_int32), ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("max_seqs", ctypes.c_int32)]


_LIB = None


def _lib():
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build the CUDA library first "
                              "(python -c 'import __graft_entry__ as g; g.build()')")
        lib = ctypes.CDLL(LIB_PATH)
        vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
        lib.kv_evict_plan.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(i64), i32,
                                      ctypes.POINTER(vp), ctypes.POINTER(ctypes.c_size_t)]
        lib.kv_evict_plan_layered.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(i64), i32, vp,
                                              ctypes.POINTER(vp), ctypes.POINTER(ctypes.c_size_t)]
        lib.kv_evict_plan_ex.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(i64), i32, vp, i32,
                                         vp, vp]
        lib.kv_evict_budget_pyramid.argtypes = [i32, i32, ctypes.c_float, vp]
        lib.kv_evict_plan_destroy.argtypes = [vp]
        lib.kv_evict_plan_destroy.restype = None
        lib.kv_evict_plan_set_debug.argtypes = [vp, ctypes.c_uint64, i32]
        lib.kv_evict_plan_set_kv_strides.argtypes = [vp, vp, vp]
        lib.kv_evict_score.argtypes = [vp] * 7
        lib.kv_evict_score_lse.argtypes = [vp] * 8
        lib.kv_evict_score_attn.argtypes = [vp] * 10
        lib.kv_evict_score_attn_workspace.argtypes = [vp, vp]
        lib.kv_evict_select.argtypes = [vp] * 11
        lib.kv_evict_select_noalloc.argtypes = [vp] * 10
        lib.kv_evict_select_profiles.argtypes = [vp, i32] + [vp] * 10
        lib.kv_evict_select_profiles_workspace.argtypes = [vp, i32, vp]
        lib.kv_evict_gather.argtypes = [vp] * 7
        lib.kv_evict_select_gather.argtypes = [vp] * 14
        lib.kv_evict_status.argtypes = [vp, vp, vp]
        lib.kv_evict_profile.argtypes = [i32, vp, i32, vp, vp]
        lib.kv_evict_cache_create.argtypes = [vp] * 7
        lib.kv_evict_cache_destroy.argtypes = [vp]
        lib.kv_evict_cache_destroy.restype = None
        lib.kv_evict_cache_reset.argtypes = [vp] * 5
        lib.kv_evict_cache_pages.argtypes = [vp] * 9 + [i64, vp, vp]
        lib.kv_evict_cache_gather.argtypes = [vp] * 5 + [i32, vp, vp, vp]
        lib.kv_evict_cache_store.argtypes = [vp] * 6 + [i64, vp, vp]
        lib.kv_evict_cache_attend.argtypes = [vp, i32, i32, i32] + [vp] * 9
        lib.kv_evict_cache_status.argtypes = [vp, vp, vp]
        lib.kv_evict_cache_append.argtypes = [vp] * 12 + [i64, vp, vp]
        lib.kv_evict_cache4_create.argtypes = [vp] * 7
        f64 = ctypes.c_double
        lib.kv_evict_rotary_frequencies.argtypes = [i32, i32] + [f64] * 5 + [vp, vp]
        lib.kv_evict_rotary_create.argtypes = [i32, i32, i32, vp, f64, vp]
        lib.kv_evict_rotary_destroy.argtypes = [vp]
        lib.kv_evict_rotary_destroy.restype = None
        lib.kv_evict_rotary_apply.argtypes = [vp] * 5 + [i32, vp, i64, i32, vp]
        lib.kv_evict_strerror.argtypes = [ctypes.c_int]
        lib.kv_evict_strerror.restype = ctypes.c_char_p
        for name in ("kv_evict_plan", "kv_evict_plan_layered", "kv_evict_plan_ex", "kv_evict_plan_set_debug",
                     "kv_evict_plan_set_kv_strides",
                     "kv_evict_score", "kv_evict_score_lse", "kv_evict_score_attn", "kv_evict_score_attn_workspace",
                     "kv_evict_select", "kv_evict_select_noalloc",
                     "kv_evict_select_profiles", "kv_evict_select_profiles_workspace", "kv_evict_gather",
                     "kv_evict_select_gather", "kv_evict_status", "kv_evict_profile",
                     "kv_evict_budget_pyramid", "kv_evict_cache_create", "kv_evict_cache_reset",
                     "kv_evict_cache_pages", "kv_evict_cache_gather", "kv_evict_cache_store",
                     "kv_evict_cache_attend", "kv_evict_cache_status", "kv_evict_cache_append", "kv_evict_cache4_create",
                     "kv_evict_rotary_frequencies", "kv_evict_rotary_create", "kv_evict_rotary_apply"):
            getattr(lib, name).restype = ctypes.c_int
        _LIB = lib
    return _LIB


def library():
    """The loaded ctypes library (loads it on first use)."""
    return _lib()


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _check(status: int, what: str):
    if status != KVE_OK:
        raise KvEvictError(status, what)


def _stream_ptr(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_config(spec: dict) -> Config:
    return Config(spec["num_layers"], spec["num_q_heads"], spec["num_kv_heads"], spec["head_dim"],
                  spec["window"], spec["budget"], spec.get("pool_kernel", 7),
                  spec.get("candidate_factor", 4), spec.get("norm_eps", 1e-12))


KVE_PLAN_PER_QUERY_HEAD = 1


class Plan:
    """kv_evict_plan (kv_evict_plan_layered when layer_budgets is given,
    kv_evict_plan_ex with KVE_PLAN_PER_QUERY_HEAD when per_query_head) for a
    configuration and the prefix lengths of the requests."""

    def __init__(self, spec: dict, seq_lens, layer_budgets=None, per_query_head: bool = False,
                 k_strides=None, v_strides=None):
        lib = _lib()
        self.spec = dict(spec)
        self.seq_lens = [int(x) for x in seq_lens]
        self._cfg = make_config(spec)
        lens = (ctypes.c_int64 * len(self.seq_lens))(*self.seq_lens)
        handle = ctypes.c_void_p()
        ws = ctypes.c_size_t()
        self.per_query_head = bool(per_query_head)
        if self.per_query_head:
            self.layer_budgets = ([int(spec["budget"])] * int(spec["num_layers"]) if layer_budgets is None
                                  else [int(b) for b in layer_budgets])
            lb = np.ascontiguousarray(self.layer_budgets, dtype=np.int32)
            _check(lib.kv_evict_plan_ex(ctypes.byref(self._cfg), lens, len(self.seq_lens), lb.ctypes.data,
                                        KVE_PLAN_PER_QUERY_HEAD, ctypes.byref(handle), ctypes.byref(ws)),
                   "kv_evict_plan_ex")
        elif layer_budgets is None:
            self.layer_budgets = [int(spec["budget"])] * int(spec["num_layers"])
            _check(lib.kv_evict_plan(ctypes.byref(self._cfg), lens, len(self.seq_lens),
                                     ctypes.byref(handle), ctypes.byref(ws)), "kv_evict_plan")
        else:
            self.layer_budgets = [int(b) for b in layer_budgets]
            lb = np.ascontiguousarray(self.layer_budgets, dtype=np.int32)
            _check(lib.kv_evict_plan_layered(ctypes.byref(self._cfg), lens, len(self.seq_lens),
                                             lb.ctypes.data, ctypes.byref(handle), ctypes.byref(ws)),
                   "kv_evict_plan_layered")
        self._h = handle
        self.workspace_bytes = ws.value
        self._kv_spans = (self._span(None),) * 2
        self._kept = {}   # kept_lens' counts by device and type
        if k_strides is not None or v_strides is not None:
            self.set_kv_strides(k_strides, v_strides)

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _LIB is not None:
            _LIB.kv_evict_plan_destroy(h)
            self._h = None

    # -- sizes of the documented layouts
    @property
    def unit_heads(self) -> int:
        """Heads per layer that own a unit: KV heads, or query heads per_query_head."""
        return self.spec["num_q_heads"] if self.per_query_head else self.spec["num_kv_heads"]

    @property
    def n_units(self) -> int:
        return len(self.seq_lens) * self.spec["num_layers"] * self.unit_heads

    @property
    def score_elems(self) -> int:
        return self.spec["num_layers"] * self.unit_heads * sum(self.seq_lens)

    def kept_lens(self, lens, first_seq: int = 0, stream=None):
        """lens (int32 [N_L, max_seqs]) with the sequences first_seq .. of this plan's requests at the rows that
        the plan keeps, min(B_l, Lc_r) + W. lens is read, and the result written, on stream. The plan's first call for
        a device copies its counts there and waits for that; later ones neither wait nor touch host memory and can
        be captured (the plan then has to live as long as the graph)."""
        import torch
        w = self.spec["window"]
        if not 0 <= first_seq <= lens.shape[1] - len(self.seq_lens):
            raise ValueError("kept_lens: the plan's requests do not fit behind first_seq")
        if isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=lens.device)
        with torch.cuda.stream(stream):   # (None changes nothing)
            kept = self._kept.get((lens.device, lens.dtype))
            if kept is None:
                kept = torch.tensor([[min(b, n - w) + w for n in self.seq_lens] for b in self.layer_budgets],
                                    dtype=lens.dtype).to(lens.device)
                self._kept[lens.device, lens.dtype] = kept
            out = lens.clone()
            out[:, first_seq:first_seq + len(self.seq_lens)] = kept
            if kept.is_cuda and not torch.cuda.is_current_stream_capturing():
                kept.record_stream(torch.cuda.current_stream(kept.device))
        return out

    def set_kv_strides(self, k_strides=None, v_strides=None):
        """kv_evict_plan_set_kv_strides: element strides (layer, KV head, token) of k
        and v, None for the dense default. For a torch tensor viewed as
        [N_L][Hkv][SL][d], pass t.stride()[:3]."""
        ks = None if k_strides is None else np.ascontiguousarray(k_strides, dtype=np.int64)
        vs = None if v_strides is None else np.ascontiguousarray(v_strides, dtype=np.int64)
        _check(_lib().kv_evict_plan_set_kv_strides(self._h, None if ks is None else ks.ctypes.data,
                                                    None if vs is None else vs.ctypes.data),
               "kv_evict_plan_set_kv_strides")
        self._kv_spans = tuple(self._span(s) for s in (ks, vs))

    def _span(self, strides):
        """(elements from the first to the last of the plan's keys or values, whether they are dense)."""
        shape = (self.spec["num_layers"], self.spec["num_kv_heads"], sum(self.seq_lens))
        if strides is None:
            return shape[0] * shape[1] * shape[2] * self.spec["head_dim"], True
        return sum((n - 1) * int(s) for n, s in zip(shape, strides)) + self.spec["head_dim"], False

    def _check_source(self, name: str, t):
        """Raises where the bf16 tensor t does not hold every row of the plan's k (name "k") or v at its strides."""
        global _bf16
        if _bf16 is None:
            import torch
            _bf16 = torch.bfloat16
        span, dense = self._kv_spans[name == "v"]
        bf16, whole = t.dtype is _bf16, t.is_contiguous()
        if bf16 and whole and t.numel() >= span:
            return
        held = 1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())) if t.numel() else 0
        if not bf16 or dense or held < span:
            raise ValueError(f"{name}: expected bf16 [num_layers, num_kv_heads, {sum(self.seq_lens)}, d], dense or with "
                             "the plan's strides")

    def set_debug(self, wait_limit_ns: int, fault: int = 0):
        _check(_lib().kv_evict_plan_set_debug(self._h, int(wait_limit_ns), int(fault)),
               "kv_evict_plan_set_debug")

    def score(self, q_win, k, mu, sigma, ws, stream=None):
        _check(_lib().kv_evict_score(self._h, _ptr(q_win), _ptr(k), _ptr(mu), _ptr(sigma), _ptr(ws),
                                     _stream_ptr(stream)), "kv_evict_score")

    def score_lse(self, q_win, k, lse, mu, sigma, ws, stream=None):
        """kv_evict_score_lse: the column pass only, given every window row's natural-log
        softmax normaliser lse (fp32, q_win's row order)."""
        _check(_lib().kv_evict_score_lse(self._h, _ptr(q_win), _ptr(k), _ptr(lse), _ptr(mu), _ptr(sigma),
                                         _ptr(ws), _stream_ptr(stream)), "kv_evict_score_lse")

    def score_attn_workspace(self) -> int:
        """Bytes of the second scratch buffer of score_attn."""
        out = ctypes.c_size_t(0)
        _check(_lib().kv_evict_score_attn_workspace(self._h, ctypes.byref(out)),
               "kv_evict_score_attn_workspace")
        return out.value

    def score_attn(self, q_win, k, v, mu, sigma, o_win, ws, attn_ws, stream=None):
        """kv_evict_score_attn: score plus the window rows' attention output o_win
        (q_win's layout, bf16)."""
        _check(_lib().kv_evict_score_attn(self._h, _ptr(q_win), _ptr(k), _ptr(v), _ptr(mu), _ptr(sigma),
                                          _ptr(o_win), _ptr(ws), _ptr(attn_ws), _stream_ptr(stream)),
               "kv_evict_score_attn")

    def select(self, mu, sigma, k, lambda1, lambda2, indices, ws, order=None, margins=None,
               stream=None):
        l1 = np.ascontiguousarray(lambda1, dtype=np.float32)
        l2 = np.ascontiguousarray(lambda2, dtype=np.float32)
        assert l1.shape == (self.spec["num_layers"],) and l2.shape == l1.shape
        _check(_lib().kv_evict_select(self._h, _ptr(mu), _ptr(sigma), _ptr(k),
                                      l1.ctypes.data, l2.ctypes.data, _ptr(indices), _ptr(order),
                                      _ptr(margins), _ptr(ws), _stream_ptr(stream)),
               "kv_evict_select")

    def select_noalloc(self, mu, sigma, k, lambda1, lambda2, indices, order=None, margins=None,
                       stream=None):
        """kv_evict_select without a workspace, for callers that cannot allocate
        device memory while they evict; its scratch is a fixed 16 MiB array inside
        the library (at most N_L * units per layer * SL = 4194304 tokens per call).
        status(None) reads its error word."""
        l1 = np.ascontiguousarray(lambda1, dtype=np.float32)
        l2 = np.ascontiguousarray(lambda2, dtype=np.float32)
        assert l1.shape == (self.spec["num_layers"],) and l2.shape == l1.shape
        _check(_lib().kv_evict_select_noalloc(self._h, _ptr(mu), _ptr(sigma), _ptr(k),
                                              l1.ctypes.data, l2.ctypes.data, _ptr(indices),
                                              _ptr(order), _ptr(margins), _stream_ptr(stream)),
               "kv_evict_select_noalloc")

    def select_profiles_workspace(self, n_profiles: int) -> int:
        """Bytes of scratch that select_profiles needs for n_profiles profiles."""
        out = ctypes.c_size_t(0)
        _check(_lib().kv_evict_select_profiles_workspace(self._h, int(n_profiles), ctypes.byref(out)),
               "kv_evict_select_profiles_workspace")
        return out.value

    def select_profiles(self, mu, sigma, k, lambda1, lambda2, indices, ws, order=None, margins=None,
                        stream=None):
        """Selection for P coefficient profiles at once: lambda1 / lambda2 are
        [P, N_L]; indices (and order / margins) are [P, n_units, B]; ws holds
        select_profiles_workspace(P) bytes."""
        l1 = np.ascontiguousarray(lambda1, dtype=np.float32)
        l2 = np.ascontiguousarray(lambda2, dtype=np.float32)
        assert l1.ndim == 2 and l1.shape[1] == self.spec["num_layers"] and l2.shape == l1.shape
        _check(_lib().kv_evict_select_profiles(self._h, int(l1.shape[0]), _ptr(mu), _ptr(sigma), _ptr(k),
                                               l1.ctypes.data, l2.ctypes.data, _ptr(indices),
                                               _ptr(order), _ptr(margins), _ptr(ws),
                                               _stream_ptr(stream)),
               "kv_evict_select_profiles")

    def gather(self, k, v, indices, k_out, v_out, stream=None):
        """kv_evict_gather. k and v may be pinned CPU tensors (read in place by the
        kernel; only the kept rows cross the host link); pageable CPU tensors are
        refused."""
        for name, t in (("k", k), ("v", v)):
            dev = getattr(t, "device", None)
            if dev is not None and getattr(dev, "type", None) == "cpu" and not t.is_pinned():
                raise ValueError(f"gather: {name} is a pageable CPU tensor; pin it or move it to the GPU")
        _check(_lib().kv_evict_gather(self._h, _ptr(k), _ptr(v), _ptr(indices), _ptr(k_out),
                                      _ptr(v_out), _stream_ptr(stream)), "kv_evict_gather")

    def select_gather(self, mu, sigma, k, v, lambda1, lambda2, indices, k_out, v_out, ws, order=None,
                      margins=None, stream=None):
        """kv_evict_select_gather: select, then the compact cache, in one launch (the
        outputs of select followed by gather). v (and k) may be pinned CPU tensors."""
        for name, t in (("k", k), ("v", v)):
            dev = getattr(t, "device", None)
            if dev is not None and getattr(dev, "type", None) == "cpu" and not t.is_pinned():
                raise ValueError(f"select_gather: {name} is a pageable CPU tensor; pin it or move it to the GPU")
        l1 = np.ascontiguousarray(lambda1, dtype=np.float32)
        l2 = np.ascontiguousarray(lambda2, dtype=np.float32)
        assert l1.shape == (self.spec["num_layers"],) and l2.shape == l1.shape
        _check(_lib().kv_evict_select_gather(self._h, _ptr(mu), _ptr(sigma), _ptr(k), _ptr(v),
                                             l1.ctypes.data, l2.ctypes.data, _ptr(indices), _ptr(order),
                                             _ptr(margins), _ptr(k_out), _ptr(v_out), _ptr(ws),
                                             _stream_ptr(stream)), "kv_evict_select_gather")

    def status(self, ws, stream=None) -> int:
        """Synchronise, return the device status (KVE_OK, KVE_ETIMEOUT or KVE_ECUDA) of
        ws and clear it; ws = None reads the error word of select_noalloc."""
        return int(_lib().kv_evict_status(self._h, _ptr(ws), _stream_ptr(stream)))


def profile(kind: str, c, num_layers: int, seg_bounds=None) -> np.ndarray:
    """Eq. 6 depth profile computed by the library (kind: global/segments/curve)."""
    k = {"global": 0, "segments": 1, "curve": 2}[kind]
    cc = np.zeros(3, dtype=np.float32)
    cc[: len(np.atleast_1d(c))] = np.atleast_1d(c)
    out = np.zeros(num_layers, dtype=np.float32)
    sb = None if seg_bounds is None else np.ascontiguousarray(seg_bounds, dtype=np.int32)
    _check(_lib().kv_evict_profile(k, cc.ctypes.data, num_layers,
                                   None if sb is None else sb.ctypes.data, out.ctypes.data),
           "kv_evict_profile")
    return out


def budget_pyramid(budget: int, num_layers: int, last_ratio: float) -> np.ndarray:
    """kv_evict_budget_pyramid: a depth-decreasing schedule with the uniform total."""
    out = np.zeros(num_layers, dtype=np.int32)
    _check(_lib().kv_evict_budget_pyramid(int(budget), int(num_layers), float(last_ratio),
                                          out.ctypes.data), "kv_evict_budget_pyramid")
    return out


class Buffers:
    """Device outputs and workspace of one call, allocated with torch."""

    def __init__(self, plan: Plan, device="cuda", with_trace: bool = True):
        import torch
        B, W, d = plan.spec["budget"], plan.spec["window"], plan.spec["head_dim"]
        n = plan.n_units
        self.mu = torch.empty(plan.score_elems, dtype=torch.float32, device=device)
        self.sigma = torch.empty_like(self.mu)
        self.indices = torch.empty((n, B), dtype=torch.int32, device=device)
        self.order = torch.empty((n, B), dtype=torch.int32, device=device) if with_trace else None
        self.margins = torch.empty((n, B), dtype=torch.float32, device=device) if with_trace else None
        self.k_out = torch.empty((n, B + W, d), dtype=torch.bfloat16, device=device)
        self.v_out = torch.empty_like(self.k_out)
        self.ws = torch.empty(plan.workspace_bytes, dtype=torch.uint8, device=device)


def run_step(plan: Plan, bufs: Buffers, q_win, k, v, lambda1, lambda2, stream=None, fused=True):
    """The whole eviction step: score, then select with the compact cache in one call
    (fused), or select and gather as two calls."""
    plan.score(q_win, k, bufs.mu, bufs.sigma, bufs.ws, stream)
    if fused:
        plan.select_gather(bufs.mu, bufs.sigma, k, v, lambda1, lambda2, bufs.indices, bufs.k_out,
                           bufs.v_out, bufs.ws, bufs.order, bufs.margins, stream)
        return
    plan.select(bufs.mu, bufs.sigma, k, lambda1, lambda2, bufs.indices, bufs.ws, bufs.order,
                bufs.margins, stream)
    plan.gather(k, v, bufs.indices, bufs.k_out, bufs.v_out, stream)


_Pair = ctypes.c_int64 * 2
_bf16 = None   # torch.bfloat16, once torch is there


def _row_strides(t, heads: int, name: str):
    """The {token, head} element strides of a bf16 tensor [..., heads, d] as a host array, or None where it
    is dense. The dimensions in front of the heads must be one run of tokens."""
    global _bf16
    if _bf16 is None:
        import torch
        _bf16 = torch.bfloat16
    shape = t.shape
    if t.dtype is not _bf16 or len(shape) < 3 or shape[-2] != heads:
        raise ValueError(f"{name}: expected bf16 [..., {heads}, d] with contiguous rows")
    if t.is_contiguous():
        return None
    st = t.stride()
    if st[-1] != 1:
        raise ValueError(f"{name}: expected bf16 [..., {heads}, d] with contiguous rows")
    if len(shape) == 3:
        return _Pair(st[0], st[1])
    token = span = None
    for i in range(len(shape) - 3, -1, -1):
        if shape[i] != 1:
            if span is None:
                token = st[i]
            elif st[i] != span:
                raise ValueError(f"{name}: its tokens are not one run")
            span = st[i] * shape[i]
    return _Pair(heads * shape[-1] if token is None else token, st[-2])


def _raw_stream(device):
    """A function that returns the address of the current stream of a CUDA device (no Stream object made: 2 us less a
    call)."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is not None and device.type == "cuda":
        index = torch.cuda.current_device() if device.index is None else device.index
        return lambda: raw(index)
    return lambda: torch.cuda.current_stream(device).cuda_stream


def _pinned(t) -> bool:
    return t.device.type == "cpu" and t.is_pinned()


def _no_gradient(call: str):
    """For a call on tensors that require a gradient: raises where autograd would have to see it."""
    import torch
    if torch.is_grad_enabled():
        raise ValueError(f"{call}: records no gradient; call it under torch.no_grad(), or from an autograd.Function whose backward "
                         "pass is rotate(..., transpose=True)")


ROTARY_KINDS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3, "yarn": 4}


class Rotary:
    """kv_evict_rotary_create: rotary positions of the first rotary_dim elements (default: all) of rows of head_dim.
    scaling names a form of kv_evict_rotary_frequencies (none, linear, ntk, parts, yarn) with its factor, original_length
    and turns (low_turns, high_turns; by default 1 and 4 for parts, 1 and 32 for yarn); frequencies (radians a position,
    rotary_dim / 2 of them) take its place where given. amplitude: what cos and sin are multiplied by (None: the
    scaling's)."""

    def __init__(self, head_dim: int = 128, rotary_dim: int | None = None, base: float = 10000.0, interleaved: bool = False,
                 scaling: str = "none", factor: float = 1.0, original_length: float = 0.0, low_turns: float = 1.0,
                 high_turns: float | None = None, frequencies=None, amplitude: float | None = None):
        import torch
        lib = _lib()
        self._h, self._i32 = None, torch.int32
        self.head_dim, self.rotary_dim = int(head_dim), int(head_dim if rotary_dim is None else rotary_dim)
        self.interleaved = bool(interleaved)
        if frequencies is None:
            if scaling not in ROTARY_KINDS:
                raise ValueError(f"scaling: one of {', '.join(ROTARY_KINDS)}")
            f = np.zeros(max(self.rotary_dim // 2, 1), dtype=np.float64)
            a = ctypes.c_double(1.0)
            high = high_turns if high_turns is not None else 32.0 if scaling == "yarn" else 4.0
            _check(lib.kv_evict_rotary_frequencies(ROTARY_KINDS[scaling], self.rotary_dim, float(base), float(factor),
                                                   float(original_length), float(low_turns), float(high), f.ctypes.data,
                                                   ctypes.byref(a)), "kv_evict_rotary_frequencies")
            amplitude = a.value if amplitude is None else amplitude
        else:
            f = np.array(frequencies, dtype=np.float64)
            if f.shape != (self.rotary_dim // 2,):
                raise ValueError("frequencies: expected rotary_dim / 2 of them")
        self.frequencies, self.amplitude = f, 1.0 if amplitude is None else float(amplitude)
        handle = ctypes.c_void_p()
        _check(lib.kv_evict_rotary_create(self.head_dim, self.rotary_dim, int(self.interleaved), f.ctypes.data,
                                          self.amplitude, ctypes.byref(handle)), "kv_evict_rotary_create")
        self._h, self._lib, self._streams = handle, lib, {}

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _LIB is not None:
            _LIB.kv_evict_rotary_destroy(h)
            self._h = None

    def rotate(self, x, positions, out=None, transpose: bool = False, stream=None):
        """kv_evict_rotary_apply: x bf16 [tokens, heads, d] (or [..., heads, d] whose tokens are one run), positions int32
        [tokens]; out, of x's shape, is returned (None: x itself, in place). A [heads, tokens, d] tensor goes in as
        x.transpose(0, 1). x and positions may lie in pinned memory. transpose: the gradient's rotation; none is recorded, and tensors that require one are refused
        where it would have to be."""
        out = x if out is None else out
        shape = x.shape
        if len(shape) < 3 or shape[-1] != self.head_dim or out.shape != shape:
            raise ValueError(f"rotate: x and out are [tokens, heads, {self.head_dim}]")
        if x.requires_grad or out.requires_grad:
            _no_gradient("rotate")
        heads, device = shape[-2], out.get_device()
        tokens = x.numel() // (heads * self.head_dim) if heads else 0
        if positions.dtype is not self._i32 or positions.numel() != tokens or not positions.is_contiguous():
            raise ValueError("rotate: positions are one contiguous int32 value a token")
        if (device < 0 or (x.get_device() != device and not _pinned(x)) or
                (positions.get_device() != device and not _pinned(positions))):
            raise ValueError("rotate: x, out and positions are on one CUDA device, x and positions there or in pinned memory")
        if stream is None:
            current = self._streams.get(device)
            if current is None:
                current = self._streams[device] = _raw_stream(out.device)
            stream = current()
        else:
            stream = _stream_ptr(stream)
        _check(self._lib.kv_evict_rotary_apply(
            self._h, x.data_ptr(), _row_strides(x, heads, "x"), out.data_ptr(), _row_strides(out, heads, "out"), heads,
            positions.data_ptr(), tokens, 1 if transpose else 0, stream), "kv_evict_rotary_apply")
        return out


class Cache8:
    """kv_evict_cache_create: the paged 8-bit cache of a configuration (num_layers, num_q_heads,
    num_kv_heads, head_dim of spec; per_query_head: the query heads are the cache's heads). Its pages
    k, v [num_pages, H, P, d] uint8 (e4m3 codes) and k_scale, v_scale [num_pages, H] fp32 are the given
    tensors, or allocated here, with the workspace ws. Tables, lengths, the free ring and slots are the
    caller's int32 tensors (state() makes them)."""

    _beside = "their scales"

    def __init__(self, spec: dict, max_seqs: int, num_pages: int, max_pages: int, page_tokens: int = 64,
                 device="cuda", per_query_head: bool = False, k=None, v=None, k_scale=None, v_scale=None):
        import torch
        heads = spec["num_q_heads"] if per_query_head else spec["num_kv_heads"]
        device = self._one_device([t for t in (k, v, k_scale, v_scale) if t is not None], device)
        shape = (num_pages, heads, page_tokens, spec["head_dim"])
        self.k, self.v = (self._buffer(t, shape, torch.uint8, device) for t in (k, v))
        self.k_scale, self.v_scale = (self._buffer(t, shape[:2], torch.float32, device) for t in (k_scale, v_scale))
        self._create("kv_evict_cache_create", spec, heads, max_seqs, num_pages, max_pages, page_tokens, self.k_scale,
                     self.v_scale)

    def _create(self, call, spec, heads, max_seqs, num_pages, max_pages, page_tokens, k_beside, v_beside):
        """The handle of the cache over its pages and what stands beside them, and the workspace."""
        import torch
        self._h = None
        self.heads = heads
        self.num_layers, self.num_q_heads, self.head_dim = spec["num_layers"], spec["num_q_heads"], spec["head_dim"]
        self.max_seqs, self.num_pages, self.max_pages, self.page_tokens = max_seqs, num_pages, max_pages, page_tokens
        if self.k.device.type != "cuda":
            raise ValueError(f"{type(self).__name__}: the pages are device memory")
        cfg = CacheConfig(self.num_layers, self.num_q_heads, self.heads, self.head_dim, page_tokens, num_pages,
                          max_pages, max_seqs)
        handle, size = ctypes.c_void_p(), ctypes.c_size_t()
        _check(getattr(_lib(), call)(ctypes.byref(cfg), _ptr(self.k), _ptr(self.v), _ptr(k_beside), _ptr(v_beside),
                                     ctypes.byref(handle), ctypes.byref(size)), call)
        self._h, self._lib = handle, _lib()
        self.ws = torch.empty(size.value, dtype=torch.uint8, device=self.k.device)
        self._ws = self.ws.data_ptr()
        self._seqs, self._entries = self.num_layers * max_seqs, self.num_layers * max_seqs * max_pages
        self._i32, self._f32 = torch.int32, torch.float32
        dev = self.k.device
        self._device = self.k.get_device()
        self._current_stream = _raw_stream(dev)
        self.reset()

    def _here(self, t) -> bool:
        """Whether kernels on the cache's device can read t."""
        return t.get_device() == self._device or _pinned(t)

    def _is_i32(self, t, n: int) -> bool:
        return (t.dtype is self._i32 and t.numel() == n and t.is_contiguous() and
                (t.get_device() == self._device or self._here(t)))

    def _stream(self, stream):
        """The stream's address; None is the current stream of the cache's device."""
        return self._current_stream() if stream is None else _stream_ptr(stream)

    @classmethod
    def _one_device(cls, given, device):
        """The device of the given pages and what stands beside them, where the others are allocated too; `device`
        where none is given."""
        if any(t.device != given[0].device for t in given):
            raise ValueError(f"{cls.__name__}: k, v and {cls._beside} are on one device")
        return given[0].device if given else device

    @staticmethod
    def _buffer(t, shape, dtype, device):
        import torch
        if t is None:
            return torch.empty(shape, dtype=dtype, device=device)
        if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
            raise ValueError(f"expected a contiguous {dtype} tensor of shape {tuple(shape)}")
        return t

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value and _LIB is not None:
            _LIB.kv_evict_cache_destroy(h)
            self._h = None

    def state(self):
        """(table, lens, free_pages, ring) of an empty cache: every page free."""
        import torch
        i32 = dict(dtype=torch.int32, device=self.k.device)
        table = torch.full((self.num_layers, self.max_seqs, self.max_pages), -1, **i32)
        lens = torch.zeros((self.num_layers, self.max_seqs), **i32)
        free, ring = torch.empty(self.num_pages, **i32), torch.empty(2, **i32)
        self.reset(free, ring)
        return table, lens, free, ring

    def reset(self, free_pages=None, ring=None, stream=None):
        """kv_evict_cache_reset: clear the workspace, and make every page free where the ring is given."""
        for name, t, n in (("free_pages", free_pages, self.num_pages), ("ring", ring, 2)):
            if t is not None and not self._is_i32(t, n):
                raise ValueError(f"{name}: expected {n} contiguous int32 values on the cache's device")
        _check(self._lib.kv_evict_cache_reset(self._h, _ptr(free_pages), _ptr(ring), self._ws,
                                              self._stream(stream)), "kv_evict_cache_reset")

    def pages(self, lens_from, lens_to, table, free_pages, ring_in, ring_out, lens_out, slots=None, stream=None):
        """kv_evict_cache_pages. slots: int32 [N_L, n] or None."""
        stride = 0
        if slots is not None:
            shape = slots.shape
            if len(shape) != 2 or shape[0] != self.num_layers or not self._is_i32(slots, shape[0] * shape[1]):
                raise ValueError("slots: expected a contiguous int32 [num_layers, n] tensor on the cache's device")
            stride = shape[1]
        seqs, i32, dev = self._seqs, self._i32, self._device
        for name, t, n in (("lens_from", lens_from, seqs), ("lens_to", lens_to, seqs), ("lens_out", lens_out, seqs),
                           ("table", table, self._entries), ("free_pages", free_pages, self.num_pages),
                           ("ring_in", ring_in, 2), ("ring_out", ring_out, 2)):
            if ((t.dtype is not i32 or t.numel() != n or t.get_device() != dev or not t.is_contiguous()) and
                    not self._is_i32(t, n)):
                raise ValueError(f"{name}: expected {n} contiguous int32 values on the cache's device")
        _check(self._lib.kv_evict_cache_pages(
            self._h, lens_from.data_ptr(), lens_to.data_ptr(), table.data_ptr(), free_pages.data_ptr(),
            ring_in.data_ptr(), ring_out.data_ptr(), lens_out.data_ptr(),
            # (an empty tensor has no address and room for no token: any address that is not NULL says so)
            None if slots is None else slots.data_ptr() or self._ws, stride, self._ws,
            self._stream(stream)), "kv_evict_cache_pages")

    def gather(self, plan: Plan, k, v, indices, table, first_seq: int = 0, stream=None):
        """kv_evict_cache_gather: the kept and the window rows of plan's requests as sequences first_seq ..;
        k and v as for Plan.gather."""
        for name, t in (("k", k), ("v", v)):
            if not self._here(t):
                raise ValueError(f"gather: {name} is on another device than the cache, or a pageable CPU tensor; move it "
                                 "to the cache's device or pin it")
            plan._check_source(name, t)
        if not self._is_i32(indices, plan.n_units * plan.spec["budget"]) or not self._is_i32(table, self._entries):
            raise ValueError("gather: indices are the plan's int32 [n_units, budget], table is int32 [num_layers, "
                             "max_seqs, max_pages]")
        _check(self._lib.kv_evict_cache_gather(self._h, plan._h, k.data_ptr(), v.data_ptr(), indices.data_ptr(),
                                               first_seq, table.data_ptr(), self._ws, self._stream(stream)),
               "kv_evict_cache_gather")

    def _check_rows(self, call, k_new, v_new, slots) -> int:
        """The tokens of a store; raises where its tensors do not hold them."""
        n = slots.numel()
        rows = n * self.heads * self.head_dim
        if k_new.numel() != rows or v_new.numel() != rows or not self._is_i32(slots, n):
            raise ValueError(f"{call}: k_new and v_new hold a row of every head for each of the int32 slots")
        if not self._here(k_new) or not self._here(v_new):
            raise ValueError(f"{call}: k_new and v_new are on the cache's device")
        return n

    def store(self, k_new, v_new, slots, stream=None):
        """kv_evict_cache_store: k_new, v_new bf16 [tokens, H, d] (slices of a projection's output too), slots
        int32 [tokens]."""
        n = self._check_rows("store", k_new, v_new, slots)
        _check(self._lib.kv_evict_cache_store(
            self._h, k_new.data_ptr(), v_new.data_ptr(), _row_strides(k_new, self.heads, "k_new"),
            _row_strides(v_new, self.heads, "v_new"), slots.data_ptr(), n, self._ws, self._stream(stream)),
            "kv_evict_cache_store")

    def append(self, rotary: Rotary, positions, k_new, v_new, slots, q=None, q_out=None, stream=None):
        """kv_evict_cache_append: store with the keys turned by positions (int32 [tokens]) on the way, and with q bf16
        [tokens, Hq, d] the queries too, into q_out (None: q itself, in place). Returns q_out."""
        n = self._check_rows("append", k_new, v_new, slots)
        if not self._is_i32(positions, n):
            raise ValueError("append: positions are one int32 value a token, on the cache's device")
        if rotary.head_dim != self.head_dim:
            raise ValueError("append: the rotation is of another head_dim than the cache")
        qs = outs = None
        if q is not None:
            q_out = q if q_out is None else q_out
            if q.numel() != n * self.num_q_heads * self.head_dim or q_out.shape != q.shape:
                raise ValueError("append: q and q_out hold a row of every query head for each token")
            if not self._here(q) or q_out.get_device() != self._device:
                raise ValueError("append: q and q_out are on the cache's device")
            if q.requires_grad or q_out.requires_grad:
                _no_gradient("append")
            qs, outs = _row_strides(q, self.num_q_heads, "q"), _row_strides(q_out, self.num_q_heads, "q_out")
        elif q_out is not None:
            raise ValueError("append: q_out without q")
        _check(self._lib.kv_evict_cache_append(
            self._h, rotary._h, positions.data_ptr(), None if q is None else q.data_ptr(), qs,
            None if q is None else q_out.data_ptr(), outs, k_new.data_ptr(), v_new.data_ptr(),
            _row_strides(k_new, self.heads, "k_new"), _row_strides(v_new, self.heads, "v_new"), slots.data_ptr(), n,
            self._ws, self._stream(stream)), "kv_evict_cache_append")
        return q_out

    def attend(self, q, table, lens, layer: int, out, lse=None, stream=None):
        """kv_evict_cache_attend: q, out bf16 [n_seq, q_tokens, Hq, d], lse fp32 [n_seq, q_tokens, Hq] or
        None; table and lens of all layers."""
        shape = q.shape
        if len(shape) != 4 or out.shape != shape or (lse is not None and (
                lse.shape != shape[:3] or lse.dtype is not self._f32 or not lse.is_contiguous())):
            raise ValueError("attend: q and out are [n_seq, q_tokens, Hq, d], lse is fp32 [n_seq, q_tokens, Hq]")
        if not self._here(q) or not self._here(out) or (lse is not None and not self._here(lse)):
            raise ValueError("attend: q, out and lse are on the cache's device")
        if not self._is_i32(table, self._entries) or not self._is_i32(lens, self._seqs):
            raise ValueError("attend: table is int32 [num_layers, max_seqs, max_pages], lens int32 [num_layers, max_seqs]")
        _check(self._lib.kv_evict_cache_attend(
            self._h, layer, shape[0], shape[1], q.data_ptr(), _row_strides(q, self.num_q_heads, "q"),
            table.data_ptr(), lens.data_ptr(), out.data_ptr(), _row_strides(out, self.num_q_heads, "out"), _ptr(lse),
            self._ws, self._stream(stream)), "kv_evict_cache_attend")

    def status(self, stream=None) -> int:
        """Synchronise, return the device status of the calls so far and clear it."""
        return int(self._lib.kv_evict_cache_status(self._h, self._ws, self._stream(stream)))


class Cache4(Cache8):
    """kv_evict_cache4_create: the paged cache in 4 bits, with the calls of Cache8. Its pages k, v [num_pages, H, P, d / 2]
    uint8 (two codes a byte) and k_param, v_param [num_pages, H, P, 2] bf16 (s and z of each row) are the given
    tensors, or allocated here."""

    _beside = "their parameters"

    def __init__(self, spec: dict, max_seqs: int, num_pages: int, max_pages: int, page_tokens: int = 64,
                 device="cuda", per_query_head: bool = False, k=None, v=None, k_param=None, v_param=None):
        import torch
        heads = spec["num_q_heads"] if per_query_head else spec["num_kv_heads"]
        device = self._one_device([t for t in (k, v, k_param, v_param) if t is not None], device)
        shape = (num_pages, heads, page_tokens)
        self.k, self.v = (self._buffer(t, shape + (spec["head_dim"] // 2,), torch.uint8, device) for t in (k, v))
        self.k_param, self.v_param = (self._buffer(t, shape + (2,), torch.bfloat16, device) for t in (k_param, v_param))
        self._create("kv_evict_cache4_create", spec, heads, max_seqs, num_pages, max_pages, page_tokens, self.k_param,
                     self.v_param)


def run_step_cache8(plan: Plan, bufs: Buffers, cache: Cache8, q_win, k, v, lambda1, lambda2, table, lens, free_pages,
                    ring, first_seq: int = 0, stream=None):
    """The eviction step whose compact cache is the paged one (a Cache8, or a Cache4): score, select, pages for the plan's
    requests (their sequences first_seq .. must be empty), and the kept and window rows written into them.
    lens and ring are advanced in place; where the free pages do not suffice, neither moves, no page is written
    and cache.status() returns KVE_EPAGES. The plan's first step on a device waits for the copy of its kept lengths
    (Plan.kept_lens); later ones do not wait and can be captured."""
    lens_to = plan.kept_lens(lens, first_seq, stream)
    plan.score(q_win, k, bufs.mu, bufs.sigma, bufs.ws, stream)
    plan.select(bufs.mu, bufs.sigma, k, lambda1, lambda2, bufs.indices, bufs.ws, bufs.order, bufs.margins, stream)
    cache.pages(lens, lens_to, table, free_pages, ring, ring, lens, None, stream)
    cache.gather(plan, k, v, bufs.indices, table, first_seq, stream)
