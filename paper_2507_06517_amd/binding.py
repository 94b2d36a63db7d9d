"""Thin ctypes binding of the C ABI in ``include/spindle.h``.

Argument marshalling only: every step of both paths runs in the HIP kernels of
``libspindle.so``.  PyTorch supplies device memory and the current HIP stream.
The raw entry points keep their C names (``spindle_compress_deep`` ...); the
``compress_deep`` / ``compress_shallow`` / ``reconstruct`` helpers allocate the
outputs and the workspace and call them.  There is no fallback: a missing
library raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libspindle.so")

F32, F16, BF16 = 0, 1, 2
NORM_PAPER, NORM_NONE = 0, 1
_DT = {"f32": F32, "f16": F16, "bf16": BF16}
E4M3, I8 = 0, 1
_FMT = {"e4m3": E4M3, "i8": I8}
HEAD_DIM = 128
_SCALE = float(np.float32(HEAD_DIM ** -0.5))

# the first N_STATUS return a status code
EXPORTS = ["spindle_deep_workspace_bytes", "spindle_compress_deep", "spindle_shallow_workspace_bytes",
           "spindle_compress_shallow", "spindle_shallow_graph", "spindle_shallow_codebook",
           "spindle_shallow_layer_workspace_bytes", "spindle_compress_shallow_layer",
           "spindle_calibrate_mfma", "spindle_calibrate_similarity", "spindle_calibrate_copy",
           "spindle_shallow_stats", "spindle_reconstruct", "spindle_profile",
           "spindle_layer_budgets", "spindle_reserve_ratio", "spindle_decode_workspace_bytes", "spindle_decode_merge",
           "spindle_decode_merge_static",
           "spindle_cache_append", "spindle_attend_workspace_bytes", "spindle_cache_attend", "spindle_cache_compact",
           "spindle_cache_copy", "spindle_pages_share", "spindle_pages_workspace_bytes", "spindle_pages_reserve",
           "spindle_pages_release",
           "spindle_profile_read", "spindle_decode_static_capacity",
           "spindle_last_error", "spindle_version"]
N_STATUS = 28


class KvDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_kv_heads", C.c_int32), ("group_size", C.c_int32),
                ("seq_len", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("stride_b", C.c_int64), ("stride_h", C.c_int64), ("stride_t", C.c_int64)]


class CacheDesc(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("n_kv_heads", C.c_int32), ("page_tokens", C.c_int32), ("head_dim", C.c_int32),
                ("format", C.c_int32), ("reserved", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("pos", C.c_void_p)]


class SpindleError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"spindle status {code}: {msg}")
        self.code = code


_lib = None


def lib():
    """Load libspindle.so (built by paper_2507_06517_amd.build); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_2507_06517_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, f32, sz = C.c_void_p, C.c_int32, C.c_float, C.c_size_t
        L.spindle_deep_workspace_bytes.argtypes = [C.POINTER(KvDesc), i32, C.POINTER(sz)]
        L.spindle_compress_deep.argtypes = [C.POINTER(KvDesc), vp, vp, vp, i32, i32, f32, i32, i32, vp, i32,
                                            vp, vp, vp, vp, vp, sz, vp]
        L.spindle_shallow_workspace_bytes.argtypes = [C.POINTER(KvDesc), i32, C.POINTER(sz)]
        for fn in (L.spindle_compress_shallow, L.spindle_shallow_graph, L.spindle_shallow_codebook):
            fn.argtypes = [C.POINTER(KvDesc), vp, vp, f32, f32, i32] + [vp] * 14 + [vp, sz, vp]
        L.spindle_shallow_layer_workspace_bytes.argtypes = [C.POINTER(KvDesc), i32, C.POINTER(sz)]
        L.spindle_compress_shallow_layer.argtypes = [C.POINTER(KvDesc), vp, vp, f32, f32, i32] + [vp] * 10 + [vp, sz, vp]
        L.spindle_calibrate_mfma.argtypes = [i32, i32, vp, C.POINTER(C.c_double)]
        L.spindle_calibrate_copy.argtypes = [vp, vp, sz, vp, C.POINTER(C.c_double)]
        L.spindle_calibrate_similarity.argtypes = [C.POINTER(KvDesc), i32, vp, sz, i32, vp, C.POINTER(C.c_double)]
        L.spindle_reconstruct.argtypes = [i32, i32, i32, i32, i32, vp, vp, vp, vp, vp]
        L.spindle_profile.argtypes = [i32]
        L.spindle_profile_read.argtypes = [C.c_char_p, C.POINTER(C.c_float), i32]
        L.spindle_profile_read.restype = C.c_int32
        L.spindle_shallow_stats.argtypes = [C.POINTER(KvDesc), i32, vp, vp, C.POINTER(C.c_int32)]
        L.spindle_layer_budgets.argtypes = [C.c_double, i32, i32, i32, C.c_double, C.POINTER(C.c_int32),
                                            C.POINTER(C.c_double)]
        L.spindle_reserve_ratio.argtypes = [C.c_int64, C.c_int64, C.c_int64, i32, i32, i32, i32, C.POINTER(C.c_double)]
        L.spindle_decode_workspace_bytes.argtypes = [C.POINTER(KvDesc), i32, C.POINTER(sz)]
        L.spindle_decode_merge.argtypes = [C.POINTER(KvDesc), vp, f32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.spindle_decode_merge_static.argtypes = [C.POINTER(KvDesc), vp, f32, i32, vp, vp, vp, vp, vp, vp, vp]
        L.spindle_decode_static_capacity.argtypes = []
        L.spindle_decode_static_capacity.restype = sz
        i64, cd = C.c_int64, C.POINTER(CacheDesc)
        L.spindle_cache_append.argtypes = [cd, vp, i32, vp, i32, vp, i32, i32, vp, vp, i32, i64, i64, i64, vp, vp]
        L.spindle_attend_workspace_bytes.argtypes = [cd, i32, i32, i32, i32, i32, i32, C.POINTER(sz)]
        L.spindle_cache_attend.argtypes = [cd, vp, i32, vp, i32, vp, i32, i32, vp, i32, i32, i64, i64, f32, f32, vp, vp, vp,
                                           vp, vp, vp, sz, vp]
        L.spindle_cache_compact.argtypes = [cd, vp, i32, vp, i32, vp, i32, vp, vp, i32, vp]
        L.spindle_cache_copy.argtypes = [cd, vp, i32, vp]
        L.spindle_pages_share.argtypes = [vp, i32, vp, vp, i32, i32, i32, vp, i32, vp, vp, vp]
        L.spindle_pages_workspace_bytes.argtypes = [i32, C.POINTER(sz)]
        L.spindle_pages_reserve.argtypes = [vp, i32, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]
        L.spindle_pages_release.argtypes = [vp, i32, vp, vp, i32, i32, i32, vp]
        for name in EXPORTS[:N_STATUS]:
            getattr(L, name).restype = C.c_int
        L.spindle_last_error.restype = C.c_char_p
        L.spindle_version.restype = C.c_uint32
        _lib = L
    return _lib


def _check(code):
    if code != 0:
        raise SpindleError(code, lib().spindle_last_error().decode())


def _ptr(t):
    """Address of a tensor as ctypes takes it for a void * (an int; None is NULL).  A c_void_p object of its own for
    each pointer of a call, and a Stream object, were 3 of the 14 us a decode call took on the host."""
    return t.data_ptr() if t is not None else None


_raw_stream = _current_device = None


def _stream():
    """Raw handle of the current stream of the current device."""
    global _raw_stream, _current_device
    if _raw_stream is None:
        import torch
        _raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
    return _raw_stream(_current_device())


def _stream_on(device):
    """_stream() for tensors of this device: kernels run on the current one and get plain addresses."""
    if device.type != "cuda":
        raise ValueError(f"the tensors are on {device}, not on a GPU")
    stream = _stream()
    if device.index != _current_device():
        raise ValueError(f"the tensors are on {device}, the current device is {_current_device()}")
    return stream


def torch_dtype(dtype: str):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def to_device(bits: np.ndarray, dtype: str, device="cuda"):
    """numpy device representation (see workloads) -> torch tensor on the GPU."""
    import torch
    if dtype == "bf16":
        return torch.from_numpy(bits.view(np.int16)).to(device).view(torch.bfloat16)
    return torch.from_numpy(bits).to(device)


def to_host_bits(t, dtype: str) -> np.ndarray:
    import torch
    if dtype == "bf16":
        return t.view(torch.int16).cpu().numpy().view(np.uint16)
    return t.cpu().numpy()


def desc_of(K, group_size: int, dtype: str) -> KvDesc:
    """Descriptor of a [B, H, l, d] tensor; a view with another memory order (say a cache stored as
    [B, l, H, d]) is described by its strides, the head dimension has to be contiguous."""
    B, H, l, d = K.shape
    if K.is_contiguous():
        return KvDesc(B, H, group_size, l, d, _DT[dtype])
    if K.stride(3) != 1:
        raise ValueError("the head dimension of K and V must be contiguous")
    return KvDesc(B, H, group_size, l, d, _DT[dtype], K.stride(0), K.stride(1), K.stride(2))


# ------------------------------------------------------------------ raw calls (same names as the C ABI)

def spindle_deep_workspace_bytes(desc: KvDesc, window: int) -> int:
    out = C.c_size_t(0)
    _check(lib().spindle_deep_workspace_bytes(C.byref(desc), window, C.byref(out)))
    return out.value


def spindle_shallow_workspace_bytes(desc: KvDesc, n_tensors: int) -> int:
    out = C.c_size_t(0)
    _check(lib().spindle_shallow_workspace_bytes(C.byref(desc), n_tensors, C.byref(out)))
    return out.value


def spindle_compress_deep(desc, K, V, Qw, window, pool_kernel, scale, norm, budget, budgets, out_stride,
                          kept_idx, K_out, V_out, scores_out, workspace, workspace_bytes, stream=None):
    _check(lib().spindle_compress_deep(C.byref(desc), _ptr(K), _ptr(V), _ptr(Qw), window, pool_kernel,
                                       float(scale), norm, budget, _ptr(budgets), out_stride, _ptr(kept_idx),
                                       _ptr(K_out), _ptr(V_out), _ptr(scores_out), _ptr(workspace),
                                       workspace_bytes, stream if stream is not None else _stream()))


def _shallow_call(fn, desc, K, V, theta_k, theta_v, max_codes, Ck, Cv, n_codes_k, n_codes_v,
                  n_found_k, n_found_v, ref_k, ref_v, mag_k, mag_v, adj_k, adj_v, deg_k, deg_v,
                  workspace, workspace_bytes, stream=None):
    _check(fn(C.byref(desc), _ptr(K), _ptr(V), float(theta_k), float(theta_v),
              max_codes, _ptr(Ck), _ptr(Cv), _ptr(n_codes_k), _ptr(n_codes_v),
              _ptr(n_found_k), _ptr(n_found_v), _ptr(ref_k), _ptr(ref_v),
              _ptr(mag_k), _ptr(mag_v), _ptr(adj_k), _ptr(adj_v), _ptr(deg_k),
              _ptr(deg_v), _ptr(workspace), workspace_bytes,
              stream if stream is not None else _stream()))


def spindle_compress_shallow(*args, **kw):
    _shallow_call(lib().spindle_compress_shallow, *args, **kw)


def spindle_shallow_graph(*args, **kw):
    """First half of spindle_compress_shallow (same arguments): up to the neighbour lists."""
    _shallow_call(lib().spindle_shallow_graph, *args, **kw)


def spindle_shallow_codebook(*args, **kw):
    """Second half of spindle_compress_shallow (same arguments, same workspace)."""
    _shallow_call(lib().spindle_shallow_codebook, *args, **kw)


def spindle_shallow_stats(desc, n_tensors, workspace, stream=None):
    """-> int32 array [units * n_tensors, 16]: rounds, entries found, exact pairs, 0, phase us..."""
    n = desc.batch * desc.n_kv_heads * n_tensors
    buf = (C.c_int32 * (16 * n))()
    _check(lib().spindle_shallow_stats(C.byref(desc), n_tensors, _ptr(workspace),
                                       stream if stream is not None else _stream(), buf))
    return np.frombuffer(buf, dtype=np.int32).reshape(n, 16).copy()


def spindle_reconstruct(units, seq_len, head_dim, dtype, max_codes, Cb, ref, mag, out, stream=None):
    _check(lib().spindle_reconstruct(units, seq_len, head_dim, dtype, max_codes, _ptr(Cb), _ptr(ref),
                                     _ptr(mag), _ptr(out), stream if stream is not None else _stream()))


def spindle_layer_budgets(reserve_ratio, seq_len, window, n_layers, beta=0.05):
    """Returns (budgets int32 [n_layers], ratios float64 [n_layers])."""
    budgets = (C.c_int32 * n_layers)()
    ratios = (C.c_double * n_layers)()
    _check(lib().spindle_layer_budgets(float(reserve_ratio), int(seq_len), int(window), int(n_layers), float(beta),
                                       budgets, ratios))
    return np.array(budgets[:], dtype=np.int32), np.array(ratios[:], dtype=np.float64)


def spindle_reserve_ratio(kept_tokens, total_tokens, codebook_entries, head_dim=128, index_bits=16, elem_bits=16,
                          magnitude_bits=32):
    """Returns (r1, r2, r3, r) of one layer; the library's magnitudes are float32."""
    out = (C.c_double * 4)()
    _check(lib().spindle_reserve_ratio(int(kept_tokens), int(total_tokens), int(codebook_entries), int(head_dim),
                                       int(index_bits), int(elem_bits), int(magnitude_bits), out))
    return tuple(out[:])


def spindle_decode_workspace_bytes(desc: KvDesc, max_codes: int) -> int:
    out = C.c_size_t(0)
    _check(lib().spindle_decode_workspace_bytes(C.byref(desc), int(max_codes), C.byref(out)))
    return out.value


def spindle_decode_merge(desc, X_new, theta, max_codes, Cb, n_codes, n_found, n_matched, ref, mag, workspace,
                         workspace_bytes, stream=None):
    _check(lib().spindle_decode_merge(C.byref(desc), _ptr(X_new), float(theta), int(max_codes), _ptr(Cb),
                                      _ptr(n_codes), _ptr(n_found), _ptr(n_matched), _ptr(ref), _ptr(mag),
                                      _ptr(workspace), int(workspace_bytes), stream or _stream()))


def spindle_decode_merge_static(desc, X_new, theta, max_codes, Cb, n_codes, n_found, n_matched, ref, mag, stream=None):
    _check(lib().spindle_decode_merge_static(C.byref(desc), _ptr(X_new), float(theta), int(max_codes), _ptr(Cb),
                                             _ptr(n_codes), _ptr(n_found), _ptr(n_matched), _ptr(ref), _ptr(mag),
                                             stream or _stream()))


def spindle_decode_static_capacity() -> int:
    return int(lib().spindle_decode_static_capacity())


def decode_merge(X_new, dtype, theta, Cb, n_codes):
    """Merges X_new [B, H, m, d] into the codebooks Cb [B, H, cap, d] (updated in place, with n_codes
    [B, H] int32).  Returns dict(ref, mag, n_found, n_matched)."""
    import torch
    B, H, m, d = X_new.shape
    desc = KvDesc(B, H, 1, m, d, _DT[dtype])
    nbytes = spindle_decode_workspace_bytes(desc, Cb.shape[2])
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=X_new.device)
    out = dict(ref=torch.empty((B, H, m), dtype=torch.int32, device=X_new.device),
               mag=torch.empty((B, H, m), dtype=torch.float32, device=X_new.device),
               n_found=torch.empty((B, H), dtype=torch.int32, device=X_new.device),
               n_matched=torch.empty((B, H), dtype=torch.int32, device=X_new.device))
    spindle_decode_merge(desc, X_new, theta, Cb.shape[2], Cb, n_codes, out["n_found"], out["n_matched"],
                         out["ref"], out["mag"], ws, ws.numel())
    out["workspace"] = ws
    return out


def spindle_profile(mode) -> None:
    """0/False: off; 1/True: HIP events around every kernel; 2: around the kernel of a codebook call that goes over all pairs."""
    _check(lib().spindle_profile(int(mode)))


def spindle_profile_read(max_records: int = 4096):
    """-> list of (kernel name, milliseconds) in launch order; clears the records."""
    names = C.create_string_buffer(32 * max_records)
    ms = (C.c_float * max_records)()
    n = lib().spindle_profile_read(names, ms, max_records)
    if n < 0:
        raise SpindleError(4, "spindle_profile_read failed")
    return [(names.raw[i * 32:(i + 1) * 32].split(b"\0", 1)[0].decode(), float(ms[i])) for i in range(n)]


# ------------------------------------------------------------------ allocating helpers

@dataclass
class DeepPlan:
    """Pre-allocated outputs and workspace of one deep call shape."""
    desc: KvDesc
    window: int
    pool: int
    scale: float
    norm: int
    budget: int
    out_stride: int
    kept: object
    K_out: object
    V_out: object
    scores: object
    ws: object
    ws_bytes: int
    budgets: object = None

    def run(self, K, V, Qw):
        spindle_compress_deep(self.desc, K, V, Qw, self.window, self.pool, self.scale, self.norm, self.budget,
                              self.budgets, self.out_stride, self.kept, self.K_out, self.V_out, self.scores,
                              self.ws, self.ws_bytes)
        return self.kept, self.K_out, self.V_out, self.scores


def plan_deep(K, group_size, dtype, window, pool, budget, scale=None, norm=NORM_PAPER, want_scores=True,
              budgets=None, out_stride=None, with_v=True) -> DeepPlan:
    import torch
    B, H, l, d = K.shape
    desc = desc_of(K, group_size, dtype)
    if scale is None:
        scale = float(np.float32(1.0 / np.sqrt(d)))
    if out_stride is None:
        out_stride = min(budget, l)
    nbytes = spindle_deep_workspace_bytes(desc, window)
    dev = K.device
    return DeepPlan(desc, window, pool, scale, norm, budget, out_stride,
                    torch.empty((B, H, out_stride), dtype=torch.int32, device=dev),
                    torch.empty((B, H, out_stride, d), dtype=K.dtype, device=dev),
                    torch.empty((B, H, out_stride, d), dtype=K.dtype, device=dev) if with_v else None,
                    torch.empty((B, H, max(l - window, 1)), dtype=torch.float32, device=dev) if want_scores else None,
                    torch.empty(nbytes, dtype=torch.uint8, device=dev), nbytes, budgets)


def compress_deep(K, V, Qw, group_size, dtype, window, pool, budget, **kw):
    plan = plan_deep(K, group_size, dtype, window, pool, budget, with_v=V is not None, **kw)
    return plan.run(K, V, Qw)


@dataclass
class ShallowPlan:
    desc: KvDesc
    theta_k: float
    theta_v: float
    max_codes: int
    out: dict
    ws: object
    ws_bytes: int

    def _args(self, K, V):
        g = self.out.get
        return (self.desc, K, V, self.theta_k, self.theta_v, self.max_codes,
                g("C_k"), g("C_v"), g("n_codes_k"), g("n_codes_v"), g("n_found_k"), g("n_found_v"),
                g("ref_k"), g("ref_v"), g("mag_k"), g("mag_v"), g("adj_k"), g("adj_v"),
                g("deg_k"), g("deg_v"), self.ws, self.ws_bytes)

    def run(self, K, V):
        spindle_compress_shallow(*self._args(K, V))
        return self.out

    def run_graph(self, K, V):
        spindle_shallow_graph(*self._args(K, V))

    def run_codebook(self, K, V):
        spindle_shallow_codebook(*self._args(K, V))
        return self.out

    def stats(self):
        n_t = sum(1 for k in self.out if k.startswith("ref_"))
        return spindle_shallow_stats(self.desc, n_t, self.ws)


def plan_shallow(K, dtype, theta_k, theta_v, max_codes, tensors=("k", "v"), debug=False) -> ShallowPlan:
    import torch
    B, H, l, d = K.shape
    desc = desc_of(K, 1, dtype)
    nbytes = spindle_shallow_workspace_bytes(desc, len(tensors))
    dev = K.device
    out = {}
    for t in tensors:
        out[f"C_{t}"] = torch.empty((B, H, max_codes, d), dtype=K.dtype, device=dev)
        out[f"n_codes_{t}"] = torch.empty((B, H), dtype=torch.int32, device=dev)
        out[f"n_found_{t}"] = torch.empty((B, H), dtype=torch.int32, device=dev)
        out[f"ref_{t}"] = torch.empty((B, H, l), dtype=torch.int32, device=dev)
        out[f"mag_{t}"] = torch.empty((B, H, l), dtype=torch.float32, device=dev)
        if debug:
            out[f"adj_{t}"] = torch.empty((B, H, l, (l + 31) // 32), dtype=torch.int32, device=dev)
            out[f"deg_{t}"] = torch.empty((B, H, l), dtype=torch.int32, device=dev)
    return ShallowPlan(desc, theta_k, theta_v, max_codes, out,
                       torch.empty(nbytes, dtype=torch.uint8, device=dev), nbytes)


class OverlappedLayer:
    """Eviction and codebook calls of one layer on two streams.  The first half of the codebook call
    (similarity graph) fills the chip; during the second half (the loop of Alg. 1, one workgroup per
    problem for most of it) most compute units are idle, so the eviction call runs beside it on a
    side stream that waits for an event recorded between the halves.  Streams and events only:
    the calls and their arguments are those of the one-stream sequence."""

    def __init__(self, deep: "DeepPlan", shallow: "ShallowPlan"):
        import torch
        self.deep, self.shallow = deep, shallow
        self.side = torch.cuda.Stream()              # default priority
        self.fork, self.join = torch.cuda.Event(), torch.cuda.Event()

    def run(self, K, V, Qw):
        import torch
        main = torch.cuda.current_stream()
        self.shallow.run_graph(K, V)
        self.fork.record(main)
        # the second half is enqueued first: its chain of short dependent kernels is the longer of
        # the two and should not queue behind an eviction kernel
        out = self.shallow.run_codebook(K, V)
        self.side.wait_event(self.fork)
        with torch.cuda.stream(self.side):
            kept = self.deep.run(K, V, Qw)
            self.join.record(self.side)
        main.wait_event(self.join)                   # later work on the main stream sees both results
        return kept, out


class PipelinedLayers:
    """Consecutive layers (independent calls) in a software pipeline over `depth` sets of buffers, each
    with a main and a side stream.  Layer k+1's similarity phase starts when layer k's has ended, so it
    runs beside layer k's codebook phase and eviction call, which leave most of the chip idle; two
    similarity phases never share the chip.  Streams and events only: every layer is the same sequence
    of calls as in OverlappedLayer, and a set's buffers are reused only after all of its work is done."""

    def __init__(self, make_plans, depth=2):
        import torch
        self.sets = []
        for _ in range(depth):
            deep, shallow = make_plans()
            self.sets.append(dict(deep=deep, shallow=shallow, main=torch.cuda.Stream(), side=torch.cuda.Stream(),
                                  graph=torch.cuda.Event(), join=torch.cuda.Event(), done=torch.cuda.Event()))
        self.k = 0
        self.prev_graph = None
        self.ready = torch.cuda.Event()

    def run(self, K, V, Qw):
        """Enqueue one layer; returns its set (outputs in set['deep'] / set['shallow'].out, valid after finish())."""
        import torch
        s = self.sets[self.k % len(self.sets)]
        self.k += 1
        main, side = s["main"], s["side"]
        self.ready.record(torch.cuda.current_stream())       # the inputs are ready on the caller's stream
        main.wait_event(self.ready)
        if self.prev_graph is not None:
            main.wait_event(self.prev_graph)                 # one similarity phase at a time
        with torch.cuda.stream(main):
            s["shallow"].run_graph(K, V)
            s["graph"].record(main)
            s["shallow"].run_codebook(K, V)
        side.wait_event(s["graph"])
        with torch.cuda.stream(side):
            s["deep"].run(K, V, Qw)
            s["join"].record(side)
        main.wait_event(s["join"])                           # the set is free again once main gets here
        s["done"].record(main)
        self.prev_graph = s["graph"]
        return s

    def finish(self):
        """The caller's stream waits for every layer enqueued so far."""
        import torch
        cur = torch.cuda.current_stream()
        for s in self.sets:
            cur.wait_event(s["done"])


def compress_shallow(K, V, dtype, theta_k, theta_v, max_codes, debug=False):
    ref = K if K is not None else V
    tensors = tuple(t for t, x in (("k", K), ("v", V)) if x is not None)
    plan = plan_shallow(ref, dtype, theta_k, theta_v, max_codes, tensors, debug)
    return plan.run(K, V)


def spindle_shallow_layer_workspace_bytes(desc: KvDesc, n_tensors: int) -> int:
    out = C.c_size_t(0)
    _check(lib().spindle_shallow_layer_workspace_bytes(C.byref(desc), int(n_tensors), C.byref(out)))
    return out.value


def spindle_compress_shallow_layer(desc, K, V, theta_k, theta_v, max_codes, Ck, Cv, n_codes_k, n_codes_v, n_found_k,
                                   n_found_v, ref_k, ref_v, mag_k, mag_v, workspace, workspace_bytes, stream=None):
    _check(lib().spindle_compress_shallow_layer(C.byref(desc), _ptr(K), _ptr(V), float(theta_k), float(theta_v),
                                                int(max_codes), _ptr(Ck), _ptr(Cv), _ptr(n_codes_k), _ptr(n_codes_v),
                                                _ptr(n_found_k), _ptr(n_found_v), _ptr(ref_k), _ptr(ref_v),
                                                _ptr(mag_k), _ptr(mag_v), _ptr(workspace), int(workspace_bytes),
                                                stream or _stream()))


def compress_shallow_layer(K, V, dtype, theta_k, theta_v, max_codes):
    """One codebook per layer over the rows of all heads.  K, V [B, H, l, d] (either may be None) ->
    dict(C_k [B, max_codes, d], n_codes_k [B], n_found_k [B], ref_k [B, H, l], mag_k [B, H, l], ... _v)."""
    import torch
    X = K if K is not None else V
    B, H, l, d = X.shape
    desc = desc_of(X, 1, dtype)
    tensors = [t for t, x in (("k", K), ("v", V)) if x is not None]
    nbytes = spindle_shallow_layer_workspace_bytes(desc, len(tensors))
    dev = X.device
    out = {}
    for t in tensors:
        out[f"C_{t}"] = torch.empty((B, max_codes, d), dtype=X.dtype, device=dev)
        out[f"n_codes_{t}"] = torch.empty((B,), dtype=torch.int32, device=dev)
        out[f"n_found_{t}"] = torch.empty((B,), dtype=torch.int32, device=dev)
        out[f"ref_{t}"] = torch.empty((B, H, l), dtype=torch.int32, device=dev)
        out[f"mag_{t}"] = torch.empty((B, H, l), dtype=torch.float32, device=dev)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    g = out.get
    spindle_compress_shallow_layer(desc, K, V, theta_k, theta_v, max_codes, g("C_k"), g("C_v"), g("n_codes_k"),
                                   g("n_codes_v"), g("n_found_k"), g("n_found_v"), g("ref_k"), g("ref_v"),
                                   g("mag_k"), g("mag_v"), ws, nbytes)
    out["workspace"] = ws
    return out


def spindle_calibrate_mfma(iters: int = 4096, pattern: int = 0, stream=None) -> float:
    """TFLOP/s of a register-resident fp16 MFMA loop on the whole chip (measurement aid); pattern 1 =
    operands with the signs and magnitudes of fp16 unit vectors."""
    out = C.c_double(0.0)
    _check(lib().spindle_calibrate_mfma(int(iters), int(pattern), stream or _stream(), C.byref(out)))
    return out.value


def spindle_calibrate_copy(src, dst, stream=None) -> float:
    """GB/s (read + written) of a plain copy of src into dst (same-size device tensors; measurement aid)."""
    out = C.c_double(0.0)
    _check(lib().spindle_calibrate_copy(_ptr(src), _ptr(dst), int(src.numel() * src.element_size()),
                                        stream or _stream(), C.byref(out)))
    return out.value


def spindle_calibrate_similarity(plan: "ShallowPlan", mode: int = 0, stream=None) -> float:
    """Milliseconds of all cosine similarities by fp16 matrix instructions, nothing done with the
    results, on stand-ins for unit vectors written to the plan's workspace (measurement aid); mode 1
    without the streaming loads, mode 2 matrix instructions only."""
    out = C.c_double(0.0)
    n_t = sum(1 for k in plan.out if k.startswith("ref_"))
    _check(lib().spindle_calibrate_similarity(C.byref(plan.desc), n_t, _ptr(plan.ws), int(plan.ws_bytes),
                                              int(mode), stream or _stream(), C.byref(out)))
    return out.value


def reconstruct(Cb, ref, mag, dtype):
    import torch
    B, H, cap, d = Cb.shape
    l = ref.shape[-1]
    out = torch.empty((B, H, l, d), dtype=Cb.dtype, device=Cb.device)
    spindle_reconstruct(B * H, l, d, _DT[dtype], cap, Cb, ref, mag, out)
    return out


# ------------------------------------------------------------------ the paged cache in 8 bits

_TORCH = {}


def _types():
    """torch's types by name, and spindle_dtype by torch type; filled at the first use."""
    if not _TORCH:
        import torch
        _TORCH.update(int32=torch.int32, uint8=torch.uint8, float32=torch.float32, empty_like=torch.empty_like, empty=torch.empty_strided,
                      codes={torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16})
    return _TORCH


def _new(shape, strides, dtype, device):
    """A new tensor with its strides given, which takes half of the time of torch.empty."""
    return _TORCH["empty"](shape, strides, dtype=_TORCH[dtype], device=device)


def _dtype_of(t):
    """spindle_dtype of a tensor of tokens."""
    code = _TORCH["codes"].get(t.dtype)
    if code is None:
        raise ValueError(f"tokens are float32, float16 or bfloat16, got {t.dtype}")
    return code


def _need(t, name, dtype, shape, device=None):
    """A contiguous tensor of this type and shape (None in the shape: any length) on the device; None passes."""
    if t is None:
        return
    if t.dtype is not _types()[dtype] or t.dim() != len(shape) or any(w is not None and w != h for w, h in zip(shape, t.shape)):
        raise ValueError(f"{name} must be {dtype} {list(shape)}, got {t.dtype} {list(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")


def _ints(t, name, shape, device):
    """_need for int32 tensors of a known shape: these checks run at every call of a decode step, so what fits passes by four
    comparisons."""
    if not (t.dtype is _TORCH["int32"] and t.shape == shape and t.device == device and t.is_contiguous()):
        _need(t, name, "int32", shape, device)


class Cache:
    """The pools of one layer: k, v uint8 [n_pages, H, page_tokens, 128], k_scale, v_scale float32 [n_pages, H], positive, and,
    optionally, pos int32 [n_pages, H, page_tokens]; format "e4m3" or "i8".  A program makes one and keeps it."""

    def __init__(self, k, v, k_scale, v_scale, pos, page_tokens, format):
        if format not in _FMT:
            raise ValueError(f"format must be one of {sorted(_FMT)}, got {format!r}")
        n_pages, heads = k.shape[:2]
        dev, size, T = k.device, (n_pages, heads, page_tokens, HEAD_DIM), _types()
        for t, name, dtype, shape in ((k, "k", "uint8", size), (v, "v", "uint8", size), (k_scale, "k_scale", "float32", size[:2]),
                                      (v_scale, "v_scale", "float32", size[:2]), (pos, "pos", "int32", size[:3])):
            if t is not None and not (t.dtype is T[dtype] and t.shape == shape and t.device == dev and t.is_contiguous()):
                _need(t, name, dtype, shape, dev)
        self.k, self.v, self.k_scale, self.v_scale, self.pos = k, v, k_scale, v_scale, pos
        self.n_pages, self.n_kv_heads, self.page_tokens, self.format = n_pages, heads, page_tokens, format
        self.desc = CacheDesc(n_pages, heads, page_tokens, HEAD_DIM, _FMT[format], 0, _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale),
                              _ptr(pos))
        self.ref = C.byref(self.desc)
        self.device = dev
        self._workspace = {}                       # bytes of cache_attend's workspace by its sizes

    def workspace_bytes(self, batch, table_width, max_q, total_q, group_size, dtype) -> int:
        key = (batch, table_width, max_q, total_q, group_size, dtype)
        n = self._workspace.get(key)
        if n is None:
            if len(self._workspace) > 4096:        # a context that grows asks for ever new sizes
                self._workspace.clear()
            n = self._workspace[key] = spindle_attend_workspace_bytes(self.ref, *key)
        return n


def new_cache(n_pages, n_kv_heads, page_tokens=64, format="e4m3", positions=False, device="cuda") -> Cache:
    import torch
    k, v = (torch.zeros((n_pages, n_kv_heads, page_tokens, HEAD_DIM), dtype=torch.uint8, device=device) for _ in range(2))
    ks, vs = (torch.zeros((n_pages, n_kv_heads), dtype=torch.float32, device=device) for _ in range(2))
    pos = torch.full((n_pages, n_kv_heads, page_tokens), -1, dtype=torch.int32, device=device) if positions else None
    return Cache(k, v, ks, vs, pos, page_tokens, format)


def spindle_cache_append(cache, table, table_width, len_, batch, cu_new, max_new, total_new, K, V, dtype, stride_b, stride_h,
                         stride_t, positions, stream=None):
    _check(lib().spindle_cache_append(cache, _ptr(table), table_width, _ptr(len_), batch, _ptr(cu_new), max_new, total_new, _ptr(K),
                                      _ptr(V), dtype, stride_b, stride_h, stride_t, _ptr(positions),
                                      stream if stream is not None else _stream()))


def spindle_attend_workspace_bytes(cache, batch, table_width, max_q, total_q, group_size, dtype) -> int:
    out = C.c_size_t(0)
    _check(lib().spindle_attend_workspace_bytes(cache, batch, table_width, max_q, total_q, group_size, dtype, C.byref(out)))
    return out.value


def spindle_cache_attend(cache, table, table_width, len_, batch, cu_q, max_q, total_q, Q, dtype, group_size, stride_t, stride_h,
                         scale, softcap, slopes, prefix, q_pos, out, lse, workspace, workspace_bytes, stream=None):
    _check(lib().spindle_cache_attend(cache, _ptr(table), table_width, _ptr(len_), batch, _ptr(cu_q), max_q, total_q, _ptr(Q), dtype,
                                      group_size, stride_t, stride_h, scale, softcap, _ptr(slopes), _ptr(prefix), _ptr(q_pos),
                                      _ptr(out), _ptr(lse), _ptr(workspace), workspace_bytes,
                                      stream if stream is not None else _stream()))


def spindle_cache_compact(cache, table, table_width, len_, batch, kept_idx, kept_stride, n_kept, table_out, out_width, stream=None):
    _check(lib().spindle_cache_compact(cache, _ptr(table), table_width, _ptr(len_), batch, _ptr(kept_idx), kept_stride, _ptr(n_kept),
                                       _ptr(table_out), out_width, stream if stream is not None else _stream()))


def spindle_cache_copy(cache, pairs, n_pairs, stream=None):
    _check(lib().spindle_cache_copy(cache, _ptr(pairs), n_pairs, stream if stream is not None else _stream()))


def spindle_pages_share(refs, n_pages, table, len_, rows_in, table_width, page_tokens, parent, rows_out, table_out, len_out,
                        stream=None):
    _check(lib().spindle_pages_share(_ptr(refs), n_pages, _ptr(table), _ptr(len_), rows_in, table_width, page_tokens, _ptr(parent),
                                     rows_out, _ptr(table_out), _ptr(len_out), stream if stream is not None else _stream()))


def spindle_pages_workspace_bytes(n_pages) -> int:
    out = C.c_size_t(0)
    _check(lib().spindle_pages_workspace_bytes(n_pages, C.byref(out)))
    return out.value


def spindle_pages_reserve(refs, n_pages, table, len_, grow, rows, table_width, page_tokens, len_out, copies, status, workspace,
                          workspace_bytes, stream=None):
    _check(lib().spindle_pages_reserve(_ptr(refs), n_pages, _ptr(table), _ptr(len_), _ptr(grow), rows, table_width, page_tokens,
                                       _ptr(len_out), _ptr(copies), _ptr(status), _ptr(workspace), workspace_bytes,
                                       stream if stream is not None else _stream()))


def spindle_pages_release(refs, n_pages, table, len_, rows, table_width, page_tokens, stream=None):
    _check(lib().spindle_pages_release(_ptr(refs), n_pages, _ptr(table), _ptr(len_), rows, table_width, page_tokens,
                                       stream if stream is not None else _stream()))


def _check_table(cache, table, lens):
    shape = table.shape
    if len(shape) != 2:
        _need(table, "table", "int32", (None, None), cache.device)
    _ints(table, "table", shape, cache.device)
    _ints(lens, "lens", shape[:1], cache.device)
    return shape


def _row_strides(t):
    """Strides of all dimensions but the last.  That of a dimension of one entry means nothing and may be anything: it is replaced
    by one that every call takes."""
    return [s if n > 1 else HEAD_DIM for s, n in zip(t.stride()[:-1], t.shape)]


def cache_append(cache: Cache, table, lens, K, V, cu_new=None, max_new=None, positions=None):
    """Stores new tokens behind the lens [B] that the sequences of table [B, width] hold.  K, V [B, H, m, d] (any order of
    the first three in memory), or, with cu_new [B + 1] int32, [tokens of all, H, d] and max_new, the most tokens of one
    sequence.  positions [tokens of all] int32.  lens is not changed.  The library takes one set of strides for K and V: where theirs
    differ, those that are not contiguous are copied."""
    B, width = _check_table(cache, table, lens)
    H, dev, shape, strides = cache.n_kv_heads, cache.device, K.shape, K.stride()
    if V.shape != shape or K.dtype is not V.dtype:
        raise ValueError("K and V must have the same type and shape")
    if K.device != dev or V.device != dev:
        raise ValueError(f"K and V are not on {dev}")
    if len(shape) != (4 if cu_new is None else 3) or shape[-1] != HEAD_DIM or strides[-1] != 1 or V.stride(-1) != 1:
        raise ValueError(f"K and V are [B, H, m, {HEAD_DIM}], or [tokens, H, {HEAD_DIM}] with cu_new, the last dimension contiguous")
    if 1 in shape or V.stride() != strides:
        strides, v_strides = _row_strides(K), _row_strides(V)
        if strides != v_strides:
            K, V = K.contiguous(), V.contiguous()
            strides = _row_strides(K)
    if cu_new is None:
        if shape[0] != B or shape[1] != H:
            raise ValueError(f"K and V must be [{B}, {H}, m, {HEAD_DIM}], got {list(shape)}")
        max_new, total = shape[2], B * shape[2]
        sb, sh, st = strides[:3]
    else:
        _ints(cu_new, "cu_new", (B + 1,), dev)
        if shape[1] != H:
            raise ValueError(f"K and V must be [tokens, {H}, {HEAD_DIM}], got {list(shape)}")
        total, sb, sh, st = shape[0], 0, strides[1], strides[0]
        max_new = total if max_new is None else int(max_new)
    if positions is not None:
        _ints(positions, "positions", (total,), dev)
    spindle_cache_append(cache.ref, table, width, lens, B, cu_new, max_new, total, K, V, _dtype_of(K), sb, sh, st, positions,
                         _stream_on(dev))


def cache_attend(cache: Cache, table, lens, Q, group_size, cu_q=None, max_q=None, scale=None, softcap=0.0, slopes=None, prefix=None,
                 q_pos=None, want_lse=False, out=None, lse=None, workspace=None):
    """Attention of the newest tokens (stored already, lens [B] counts them) over their sequences.  Q [B, m, H * group, d]
    (the tokens of all sequences at one stride), or, with cu_q [B + 1] int32, [tokens of all, H * group, d] and max_q, the most tokens
    of one sequence.  Returns out, or (out, lse) with want_lse; out, lse and
    workspace may be passed in (a workspace of spindle_attend_workspace_bytes,
    contiguous).  Rows of Q that are no sequence's, by cu_q, get nothing."""
    B, width = _check_table(cache, table, lens)
    dev, hq, shape, strides = cache.device, cache.n_kv_heads * group_size, Q.shape, Q.stride()
    if len(shape) != (4 if cu_q is None else 3) or shape[-1] != HEAD_DIM or shape[-2] != hq or strides[-1] != 1 or Q.device != dev:
        raise ValueError(f"Q is [B, m, {hq}, {HEAD_DIM}], or [tokens, {hq}, {HEAD_DIM}] with cu_q, on {dev}, the last dimension contiguous")
    if cu_q is None:
        if shape[0] != B:
            raise ValueError(f"Q has {shape[0]} sequences, table {B}")
        max_q, total = shape[1], B * shape[1]
        st = strides[0 if max_q == 1 else 1]       # (with one token a sequence the next token is the next sequence's)
        if max_q > 1 and B > 1 and strides[0] != max_q * st:
            raise ValueError("the tokens of all sequences must follow each other at one stride")
    else:
        _ints(cu_q, "cu_q", (B + 1,), dev)
        total, st = shape[0], strides[0]
        max_q = total if max_q is None else int(max_q)
    # the stride of a dimension of one entry means nothing, and may be anything
    if total < 2:
        st = HEAD_DIM
    sh = HEAD_DIM if hq == 1 else strides[-2]
    if slopes is not None:
        _need(slopes, "slopes", "float32", (hq,), dev)
    if prefix is not None:
        _ints(prefix, "prefix", (B,), dev)
    if q_pos is not None:
        _ints(q_pos, "q_pos", (total,), dev)
    dt = _dtype_of(Q)
    if out is None:
        out = _TORCH["empty_like"](Q) if Q.is_contiguous() else Q.new_empty(shape)
    elif out.shape != shape or out.dtype is not Q.dtype or not out.is_contiguous() or out.device != dev:
        raise ValueError("out must be a contiguous tensor of Q's type and shape")
    if lse is not None:
        _need(lse, "lse", "float32", tuple(shape[:-1]), dev)
    elif want_lse:
        lse = _new(shape[:-1], (hq, 1) if cu_q is not None else (max_q * hq, hq, 1), "float32", dev)
    if workspace is None:
        nbytes = cache.workspace_bytes(B, width, max_q, total, group_size, dt)
        if nbytes:
            workspace = _new((nbytes,), (1,), "uint8", dev)
    else:
        if workspace.device != dev or not workspace.is_contiguous():
            raise ValueError(f"workspace must be a contiguous tensor on {dev}")
        nbytes = workspace.numel() * workspace.element_size()
    spindle_cache_attend(cache.ref, table, width, lens, B, cu_q, max_q, total, Q, dt, group_size, st, sh,
                         _SCALE if scale is None else scale, softcap, slopes, prefix, q_pos, out, lse, workspace, nbytes,
                         _stream_on(dev))
    return out if lse is None else (out, lse)


def cache_compact(cache: Cache, table, lens, kept, n_kept, table_out):
    """Gathers the tokens kept [B, H, stride] int32 (as compress_deep returns them), n_kept [B] of each head, into the pages of
    table_out [B, width_out]."""
    B, width = _check_table(cache, table, lens)
    dev, stride, width_out = cache.device, kept.shape[-1], table_out.shape[-1]
    _ints(kept, "kept", (B, cache.n_kv_heads, stride), dev)
    _ints(n_kept, "n_kept", (B,), dev)
    _ints(table_out, "table_out", (B, width_out), dev)
    spindle_cache_compact(cache.ref, table, width, lens, B, kept, stride, n_kept, table_out, width_out, _stream_on(dev))


def cache_copy(cache: Cache, copies):
    """Copies pages, copies [n, 2] int32 (from, to); -1 copies nothing."""
    n = copies.shape[0]
    _ints(copies, "copies", (n, 2), cache.device)
    spindle_cache_copy(cache.ref, copies, n, _stream_on(cache.device))


def _check_pages(refs, table, lens):
    dev, shape, n_pages = refs.device, table.shape, refs.shape[0]
    if len(shape) != 2 or not _TORCH:
        _need(table, "table", "int32", (None, None), dev)
    _ints(refs, "refs", (n_pages,), dev)
    _ints(table, "table", shape, dev)
    _ints(lens, "lens", shape[:1], dev)
    return dev, shape[0], shape[1], n_pages


def pages_share(refs, table, lens, parent, page_tokens):
    """Row r of the result holds the pages of row parent[r] (-1: none).  Returns (table_out, lens_out)."""
    dev, rows_in, width, n_pages = _check_pages(refs, table, lens)
    rows = parent.shape[0]
    _ints(parent, "parent", (rows,), dev)
    out, n = _new((rows, width), (width, 1), "int32", dev), _new((rows,), (1,), "int32", dev)
    spindle_pages_share(refs, n_pages, table, lens, rows_in, width, page_tokens, parent, rows, out, n, _stream_on(dev))
    return out, n


def pages_reserve(refs, table, lens, grow, page_tokens):
    """Pages for grow [B] more tokens of each row; table is changed in place.  Returns (lens_out [B], copies [B, 2], status [2]);
    the copies are cache_copy's to make, in every layer that the table serves."""
    dev, rows, width, n_pages = _check_pages(refs, table, lens)
    _ints(grow, "grow", (rows,), dev)
    n, copies, status = _new((rows,), (1,), "int32", dev), _new((rows, 2), (2, 1), "int32", dev), _new((2,), (1,), "int32", dev)
    nws = (n_pages + 63) // 64 * 64                # spindle_pages_workspace_bytes in ints
    ws = _new((nws,), (1,), "int32", dev)
    spindle_pages_reserve(refs, n_pages, table, lens, grow, rows, width, page_tokens, n, copies, status, ws, 4 * nws, _stream_on(dev))
    return n, copies, status


def pages_release(refs, table, lens, page_tokens):
    """The rows' pages are held once less."""
    dev, rows, width, n_pages = _check_pages(refs, table, lens)
    spindle_pages_release(refs, n_pages, table, lens, rows, width, page_tokens, _stream_on(dev))
