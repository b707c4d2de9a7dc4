"""ctypes binding of libtcuscan.so -- argument marshalling only.

Same names as the C entry points in ``include/tcuscan.h``.  Tensors are torch CUDA tensors
(PyTorch is used for device memory and streams, nothing else); every step of the scan runs in
the HIP kernels.  There is no CPU fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtcuscan.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP = 0, 1, 2, 3, 4
I32_I32, F16_F32, I8_I32, F32_F32, BF16_F32 = 0, 1, 2, 3, 4
DTYPES = {"i32": I32_I32, "f16": F16_F32, "i8": I8_I32, "f32": F32_F32, "bf16": BF16_F32}

EXPORTS = ["tcuscan_workspace_bytes", "tcuscan_workspace_init", "tcuscan_inclusive", "tcuscan_exclusive",
           "tcuscan_batched", "tcuscan_scan", "tcuscan_segmented_workspace_bytes", "tcuscan_segmented", "tcuscan_tile_elems", "tcuscan_large_tile_elems", "tcuscan_huge_tile_elems",
           "tcuscan_set_tile_policy", "tcuscan_set_segmented_form",
           "tcuscan_workspace_fault", "tcuscan_matmulscan_levels", "tcuscan_matmulscan_levels_radix", "tcuscan_compact_u32",
           "tcuscan_split_radix_sort_u32", "tcuscan_set_sort_fusion", "tcuscan_status_string",
           "tcuscan_set_chain_policy", "tcuscan_scan_static", "tcuscan_path_for", "tcuscan_measure_stream",
           "tcuscan_test_advance_calls", "tcuscan_test_tag_period", "tcuscan_test_chain_fault",
           "tcuscan_decay_attention_workspace_bytes", "tcuscan_decay_attention", "tcuscan_decay_attention_backward",
           "tcuscan_decay_attention_step", "tcuscan_embedding", "tcuscan_embedding_backward_workspace_bytes", "tcuscan_embedding_backward"]

_lib = None


class TcuscanError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} (status {code})")


def load() -> ctypes.CDLL:
    """Load the built library.  Building is a separate step (``python -m paper_2411_17887_amd.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not built; run `python -m paper_2411_17887_amd.build` (hipcc, gfx950)")
        # PyTorch ships its own HIP runtime; it must be the one already mapped when this library's
        # dependency on libamdhip64 is resolved, or the process ends up with two runtimes that do not
        # know each other's streams and allocations.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        L.tcuscan_workspace_bytes.argtypes = [sz, sz, ci]
        L.tcuscan_workspace_bytes.restype = sz
        L.tcuscan_tile_elems.argtypes = [ci]
        L.tcuscan_tile_elems.restype = sz
        L.tcuscan_large_tile_elems.argtypes = [ci]
        L.tcuscan_large_tile_elems.restype = sz
        L.tcuscan_huge_tile_elems.argtypes = [ci]
        L.tcuscan_huge_tile_elems.restype = sz
        L.tcuscan_set_tile_policy.argtypes = [ci]
        L.tcuscan_set_tile_policy.restype = ci
        L.tcuscan_set_sort_fusion.argtypes = [ci]
        L.tcuscan_set_sort_fusion.restype = ci
        L.tcuscan_set_segmented_form.argtypes = [ci]
        L.tcuscan_set_segmented_form.restype = ci
        L.tcuscan_workspace_init.argtypes = [vp, sz, vp]
        L.tcuscan_inclusive.argtypes = [vp, vp, sz, ci, vp, sz, vp]
        L.tcuscan_exclusive.argtypes = [vp, vp, sz, ci, vp, sz, vp]
        L.tcuscan_batched.argtypes = [vp, vp, sz, sz, ci, ci, vp, sz, vp]
        L.tcuscan_scan.argtypes = [vp, vp, sz, sz, ci, ctypes.c_uint, vp, sz, vp]
        L.tcuscan_segmented_workspace_bytes.argtypes = [sz, sz, ci]
        L.tcuscan_segmented_workspace_bytes.restype = sz
        L.tcuscan_segmented.argtypes = [vp, vp, vp, sz, sz, ci, ctypes.c_uint, vp, sz, vp]
        L.tcuscan_workspace_fault.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_uint)]
        L.tcuscan_matmulscan_levels.argtypes = [vp, vp, sz, ci, ci, vp, vp]
        L.tcuscan_matmulscan_levels_radix.argtypes = [vp, vp, sz, ci, ci, ci, vp, vp]
        L.tcuscan_compact_u32.argtypes = [vp, vp, vp, sz, vp, vp, vp, sz, vp]
        L.tcuscan_split_radix_sort_u32.argtypes = [vp, vp, sz, ci, vp, vp, vp, vp, vp, sz, vp]
        L.tcuscan_set_chain_policy.argtypes = [ci]
        L.tcuscan_set_chain_policy.restype = ci
        L.tcuscan_scan_static.argtypes = [vp, vp, sz, sz, ci, ctypes.c_uint, vp]
        L.tcuscan_scan_static.restype = ci
        L.tcuscan_path_for.argtypes = [vp, sz, sz, ci, sz]
        L.tcuscan_path_for.restype = ci
        L.tcuscan_measure_stream.argtypes = [vp, vp, sz, ci, ctypes.c_uint, vp]
        L.tcuscan_measure_stream.restype = ci
        L.tcuscan_test_advance_calls.argtypes = [ctypes.c_ulonglong]
        L.tcuscan_test_advance_calls.restype = ci
        L.tcuscan_test_tag_period.argtypes = []
        L.tcuscan_test_tag_period.restype = ctypes.c_ulonglong
        L.tcuscan_test_chain_fault.argtypes = [ctypes.c_uint, ctypes.c_longlong]
        L.tcuscan_test_chain_fault.restype = ci
        L.tcuscan_status_string.argtypes = [ci]
        L.tcuscan_status_string.restype = ctypes.c_char_p
        cf, ll = ctypes.c_float, ctypes.c_longlong
        L.tcuscan_decay_attention_workspace_bytes.argtypes = [vp, ci, ci]
        L.tcuscan_decay_attention_workspace_bytes.restype = sz
        L.tcuscan_decay_attention.argtypes = [vp] * 7 + [ci, cf, vp, vp, vp, sz, vp, sz, vp]
        L.tcuscan_decay_attention_backward.argtypes = [vp] * 10 + [ci, cf, vp, vp, vp, vp, sz, vp]
        L.tcuscan_decay_attention_step.argtypes = [vp] * 6 + [ci, cf, vp, vp, sz, vp, sz, vp]
        L.tcuscan_embedding.argtypes = [vp, ci, sz, vp, sz, sz, sz, ci, vp, sz, ci, cf, vp, sz, vp]
        L.tcuscan_embedding_backward_workspace_bytes.argtypes = [sz, sz, sz]
        L.tcuscan_embedding_backward_workspace_bytes.restype = sz
        L.tcuscan_embedding_backward.argtypes = [vp, ci, sz, vp, sz, ci, vp, sz, sz, sz, ci, cf, ll, ctypes.c_uint, vp, sz, vp]
        for f in ("tcuscan_decay_attention", "tcuscan_decay_attention_backward", "tcuscan_decay_attention_step", "tcuscan_embedding",
                  "tcuscan_embedding_backward", "tcuscan_workspace_init", "tcuscan_inclusive", "tcuscan_exclusive", "tcuscan_batched", "tcuscan_scan", "tcuscan_segmented",
                  "tcuscan_workspace_fault", "tcuscan_matmulscan_levels", "tcuscan_matmulscan_levels_radix",
                  "tcuscan_compact_u32", "tcuscan_split_radix_sort_u32"):
            getattr(L, f).restype = ci
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return load().tcuscan_status_string(int(code)).decode()


def _dt(dt) -> int:
    return DTYPES[dt] if isinstance(dt, str) else int(dt)


def workspace_bytes(rows: int, cols: int, dt) -> int:
    return int(load().tcuscan_workspace_bytes(rows, cols, _dt(dt)))


def tile_elems(dt) -> int:
    return int(load().tcuscan_tile_elems(_dt(dt)))


def large_tile_elems(dt) -> int:
    return int(load().tcuscan_large_tile_elems(_dt(dt)))


def huge_tile_elems(dt) -> int:
    return int(load().tcuscan_huge_tile_elems(_dt(dt)))


TILE_AUTO, TILE_SMALL, TILE_LARGE, TILE_HUGE = 0, 1, 2, 3


def set_tile_policy(policy: int) -> None:
    rc = load().tcuscan_set_tile_policy(int(policy))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_set_tile_policy")


def _stream(stream) -> int:
    if stream is None:
        # the current stream of the current device, without the object around it: 0.4 us where
        # torch.cuda.current_stream() takes 2.9 of the 6.9 that a small call took in all
        import torch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return int(getattr(stream, "cuda_stream", stream))


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _ws_args(ws):
    return (_ptr(ws), 0 if ws is None else ws.numel() * ws.element_size())


def new_workspace(rows: int, cols: int, dt, device="cuda"):
    """Allocate and zero a workspace tensor (None when the shape needs none)."""
    import torch
    nbytes = workspace_bytes(rows, cols, dt)
    if nbytes == 0:
        return None
    return torch.zeros((nbytes + 7) // 8, dtype=torch.int64, device=device)


def workspace_init(ws, stream=None) -> None:
    p, nb = _ws_args(ws)
    rc = load().tcuscan_workspace_init(p, nb, _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_workspace_init")


def inclusive(x, out, dt, ws=None, stream=None, n=None) -> None:
    rc = load().tcuscan_inclusive(_ptr(x), _ptr(out), x.numel() if n is None else n, _dt(dt), *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_inclusive")


def exclusive(x, out, dt, ws=None, stream=None, n=None) -> None:
    rc = load().tcuscan_exclusive(_ptr(x), _ptr(out), x.numel() if n is None else n, _dt(dt), *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_exclusive")


def batched(x, out, rows: int, cols: int, dt, exclusive_scan: bool = False, ws=None, stream=None) -> None:
    rc = load().tcuscan_batched(_ptr(x), _ptr(out), rows, cols, _dt(dt), int(bool(exclusive_scan)), *_ws_args(ws),
                                _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_batched")


EXCLUSIVE, REVERSE = 1, 2      # flag bits of tcuscan_scan


def scan(x, out, rows: int, cols: int, dt, flags: int = 0, ws=None, stream=None) -> None:
    """Row-wise scans with option flags (EXCLUSIVE, REVERSE = suffix sums)."""
    rc = load().tcuscan_scan(_ptr(x), _ptr(out), rows, cols, _dt(dt), int(flags), *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_scan")


def segmented_workspace_bytes(rows: int, total: int, dt) -> int:
    return int(load().tcuscan_segmented_workspace_bytes(rows, total, _dt(dt)))


def new_segmented_workspace(rows: int, total: int, dt):
    """A zero-filled workspace for tcuscan_segmented (None when nothing is to be done)."""
    import torch
    nbytes = segmented_workspace_bytes(rows, total, dt)
    return torch.zeros(nbytes // 8 + 1, dtype=torch.int64, device="cuda") if nbytes else None


def segmented(x, out, offsets, rows: int, total: int, dt, flags: int = 0, ws=None, stream=None) -> None:
    """Row-wise scans of rows stored back to back; `offsets`: int64 device tensor of rows + 1 element offsets."""
    rc = load().tcuscan_segmented(_ptr(x), _ptr(out), _ptr(offsets), rows, total, _dt(dt), int(flags), *_ws_args(ws),
                                  _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_segmented")


def matmulscan_levels(x, out, dt, rounds: int = -1, matmuls=None, stream=None, n=None, s: int = 16) -> None:
    """Algorithm 1 round by round (n = s^k; s = 16 by default, 4 and 32 as well).  `matmuls`: optional int64
    device tensor of one element."""
    n = x.numel() if n is None else n
    if s == 16:
        rc = load().tcuscan_matmulscan_levels(_ptr(x), _ptr(out), n, _dt(dt), int(rounds), _ptr(matmuls), _stream(stream))
    else:
        rc = load().tcuscan_matmulscan_levels_radix(_ptr(x), _ptr(out), n, _dt(dt), int(s), int(rounds), _ptr(matmuls),
                                                    _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_matmulscan_levels")


def compact_u32(values, mask, out, positions, count=None, ws=None, stream=None) -> None:
    """out <- values[mask != 0] in order; positions (int32, n) is scratch; count: optional 1-element int32 tensor."""
    rc = load().tcuscan_compact_u32(_ptr(values), _ptr(mask), _ptr(out), values.numel(), _ptr(positions), _ptr(count),
                                    *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_compact_u32")


def set_segmented_form(flat: bool) -> None:
    load().tcuscan_set_segmented_form(int(bool(flat)))


def set_sort_fusion(form: int) -> None:
    """1: passes on eight bits (default); 2: fused passes on one bit; 0: mask kernel + scan + scatter kernel."""
    rc = load().tcuscan_set_sort_fusion(int(form))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_set_sort_fusion")


def split_radix_sort_u32(keys, keys_tmp, flags, positions, vals=None, vals_tmp=None, bits: int = 32, ws=None, stream=None) -> None:
    """Stable radix sort of 32-bit keys (and optional payloads) by their low `bits` bits: passes on up to eight bits, or fewer of them and a workgroup
    per bucket (set_sort_fusion: one bit per pass)."""
    rc = load().tcuscan_split_radix_sort_u32(_ptr(keys), _ptr(vals), keys.numel(), int(bits), _ptr(keys_tmp), _ptr(vals_tmp),
                                             _ptr(flags), _ptr(positions), *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_split_radix_sort_u32")


STATIC_SCRATCH = "static"      # workspace_fault(STATIC_SCRATCH): the fixed scratch of scan_static on the current GPU
STATIC_SCRATCH_BYTES = 4194560
PATH_ROWS, PATH_TILES, PATH_TILES_FROM_BOUNDARY, PATH_ELEMENTWISE = 0, 1, 2, 3


def scan_static(x, out, rows: int, cols: int, dt, flags: int = 0, stream=None) -> None:
    """tcuscan_scan without a workspace argument: the library's fixed device scratch is used; allocates nothing."""
    rc = load().tcuscan_scan_static(_ptr(x), _ptr(out), rows, cols, _dt(dt), int(flags), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_scan_static")


def path_for(in_ptr: int, rows: int, cols: int, dt, ws_bytes: int) -> int:
    return int(load().tcuscan_path_for(int(in_ptr), rows, cols, _dt(dt), ws_bytes))


def set_chain_policy(policy: int) -> None:
    """0: tiles in workgroup-index order (default); 1: tiles drawn from a ticket counter."""
    rc = load().tcuscan_set_chain_policy(int(policy))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_set_chain_policy")


def measure_stream(x, out, out_bytes: int, in_bytes_per_out_word: int, variant: int = 0, stream=None) -> None:
    """The streaming yardstick kernel (measurement only)."""
    rc = load().tcuscan_measure_stream(_ptr(x), _ptr(out), out_bytes, int(in_bytes_per_out_word), int(variant), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_measure_stream")


def test_advance_calls(calls: int) -> None:
    load().tcuscan_test_advance_calls(int(calls))


def test_tag_period() -> int:
    return int(load().tcuscan_test_tag_period())


def test_chain_fault(spin_limit: int = 0, mute_tile: int = -1) -> None:
    rc = load().tcuscan_test_chain_fault(int(spin_limit), int(mute_tile))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_test_chain_fault")


def workspace_fault(ws, stream=None) -> int:
    v = ctypes.c_uint(0)
    rc = load().tcuscan_workspace_fault(1 if isinstance(ws, str) and ws == STATIC_SCRATCH else _ptr(ws), _stream(stream), ctypes.byref(v))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_workspace_fault")
    return int(v.value)


# ---- operators on tokens: linear attention with decays, embeddings

ACCUMULATE = 1                 # flag bit of tcuscan_embedding_backward
_ELEMENTS = {}                 # torch.dtype -> the dtype whose input it is
_pack_shape = struct.Struct("22q").pack


def _element(t) -> int:
    if not _ELEMENTS:
        import torch
        _ELEMENTS.update({torch.float16: F16_F32, torch.bfloat16: BF16_F32, torch.float32: F32_F32})
    return _ELEMENTS.get(t.dtype, -1)


def _refuse(condition, what: str) -> None:
    if condition:
        raise ValueError(what)


def _attention_shape(rows, q, k, v, out, log_decay, dq=None, dk=None, dv=None) -> tuple[bytes, int]:
    """The C call's shape and element type, from tensors [token, stored head, feature]."""
    (total, q_heads, d_k), (k_total, k_heads, k_dim), (v_total, v_heads, d_v), (o_total, heads, o_dim) = q.shape, k.shape, v.shape, out.shape
    _refuse(not total == k_total == v_total == o_total, "q, k, v and out have different numbers of tokens")
    _refuse(d_k != k_dim or d_v != o_dim or log_decay.numel() != heads, "features of q and k, of v and out, or heads of out and decays differ")
    dt = q.dtype
    _refuse(not dt == k.dtype == v.dtype == out.dtype, "q, k, v and out have different types")
    (qt, qh, q1), (kt, kh, k1), (vt, vh, v1), (ot, oh, o1) = q.stride(), k.stride(), v.stride(), out.stride()
    _refuse((q1 != 1 or k1 != 1) and d_k > 1 or (v1 != 1 or o1 != 1) and d_v > 1, "features have to be dense")
    grads = (0, 0, 0, 0, 0, 0)
    if dq is not None:
        for g, x in ((dq, q), (dk, k), (dv, v)):
            _refuse(g.shape != x.shape or g.dtype != dt or g.stride(2) != 1 and g.shape[2] > 1, "a gradient's shape, type or stride is not its input's")
        grads = (*dq.stride()[:2], *dk.stride()[:2], *dv.stride()[:2])
    return _pack_shape(rows, total, heads, d_k, d_v, q_heads, k_heads, v_heads, qt, qh, kt, kh, vt, vh, ot, oh, *grads), _element(q)


def _check_states(states, heads: int, d_k: int, d_v: int) -> int:
    """[states, heads, dk, dv] of fp32, dense.  Returns how many there are."""
    import torch
    _refuse(states.dtype != torch.float32 or states.shape[1:] != (heads, d_k, d_v) or not states.is_contiguous(),
            "states are dense fp32 tensors [states, heads, dk, dv]")
    return states.shape[0]


def _check_longs(t, n: int, what: str) -> None:
    import torch
    _refuse(t.dtype != torch.int64 or t.numel() != n or not t.is_contiguous(), f"{what}: a dense int64 tensor of {n} elements is wanted")


def _check_decays(t) -> None:
    import torch
    _refuse(t.dtype != torch.float32 or not t.is_contiguous(), "log_decay: a dense fp32 tensor is wanted")


def _zeros(nbytes: int):
    import torch
    return torch.zeros((nbytes + 7) // 8, dtype=torch.int64, device="cuda")


def decay_attention_workspace_bytes(rows: int, total: int, heads: int, d_k: int, d_v: int, q_heads=None, k_heads=None, v_heads=None, dt="bf16",
                                    backward: bool = False) -> int:
    shape = _pack_shape(rows, total, heads, d_k, d_v, q_heads or heads, k_heads or heads, v_heads or heads, *[0] * 14)
    return int(load().tcuscan_decay_attention_workspace_bytes(shape, _dt(dt), int(backward)))


def new_decay_attention_workspace(rows: int, total: int, heads: int, d_k: int, d_v: int, q_heads=None, k_heads=None, v_heads=None, dt="bf16"):
    """A zero-filled workspace for decay_attention on up to `rows` rows of `total` tokens in all."""
    return _zeros(decay_attention_workspace_bytes(rows, total, heads, d_k, d_v, q_heads, k_heads, v_heads, dt))


def new_decay_attention_backward_workspace(rows: int, total: int, heads: int, d_k: int, d_v: int, q_heads=None, k_heads=None, v_heads=None,
                                           dt="bf16"):
    """The same for decay_attention_backward; q_heads, k_heads and v_heads where fewer are stored than `heads`."""
    return _zeros(decay_attention_workspace_bytes(rows, total, heads, d_k, d_v, q_heads, k_heads, v_heads, dt, backward=True))


def decay_attention(q, k, v, out, log_decay, offsets, scale: float = 1.0, state_in=None, state_out=None, slots=None, ws=None, stream=None) -> None:
    """Linear attention with one decay per head over rows of tokens stored back to back.

    q [total, q_heads, dk], k [total, k_heads, dk], v [total, v_heads, dv], out [total, heads, dv]: any strides, features dense;
    log_decay [heads]; offsets int64 [rows + 1]; state_in, state_out [states, heads, dk, dv] fp32 or None; slots int64 [rows] or None."""
    rows = offsets.numel() - 1
    shape, dt = _attention_shape(rows, q, k, v, out, log_decay)
    _check_decays(log_decay)
    _check_longs(offsets, rows + 1, "offsets")
    states = 0
    for t in (state_in, state_out):
        if t is not None:
            n = _check_states(t, out.shape[1], q.shape[2], v.shape[2])
            _refuse(states and n != states, "state_in and state_out hold different numbers of states")
            states = n
    if slots is not None:
        _check_longs(slots, rows, "slots")
    rc = load().tcuscan_decay_attention(shape, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), log_decay.data_ptr(), offsets.data_ptr(), dt, scale,
                                        _ptr(state_in), _ptr(state_out), _ptr(slots), states, *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_decay_attention")


def decay_attention_backward(q, k, v, d_out, dq, dk, dv, log_decay, offsets, scale: float = 1.0, state_in=None, d_state_out=None, d_state_in=None,
                             ws=None, stream=None) -> None:
    """The gradients by q, k, v (into dq, dk, dv) and by state_in (into d_state_in, if given) from those by out and by state_out."""
    rows = offsets.numel() - 1
    shape, dt = _attention_shape(rows, q, k, v, d_out, log_decay, dq, dk, dv)
    _check_decays(log_decay)
    _check_longs(offsets, rows + 1, "offsets")
    for t in (state_in, d_state_out, d_state_in):
        if t is not None:
            _refuse(_check_states(t, d_out.shape[1], q.shape[2], v.shape[2]) != rows, "a state for each row is wanted")
    rc = load().tcuscan_decay_attention_backward(shape, q.data_ptr(), k.data_ptr(), v.data_ptr(), d_out.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
                                                 log_decay.data_ptr(), offsets.data_ptr(), dt, scale, _ptr(state_in), _ptr(d_state_out), _ptr(d_state_in),
                                                 *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_decay_attention_backward")


def decay_attention_step(q, k, v, out, log_decay, state, slots=None, scale: float = 1.0, ws=None, stream=None) -> None:
    """One token for each of n sequences: q [n, q_heads, dk], ..., out [n, heads, dv]; state [states, heads, dk, dv] fp32, updated in
    place where slots (int64 [n], None: 0 .. n - 1) point."""
    n = q.shape[0]
    shape, dt = _attention_shape(n, q, k, v, out, log_decay)
    _check_decays(log_decay)
    states = _check_states(state, out.shape[1], q.shape[2], v.shape[2])
    if slots is not None:
        _check_longs(slots, n, "slots")
    rc = load().tcuscan_decay_attention_step(shape, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), log_decay.data_ptr(), dt, scale, state.data_ptr(),
                                             _ptr(slots), states, *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_decay_attention_step")


def _check_tokens(ids, rows, table) -> None:
    """ids: n dense integers of 4 or 8 bytes; rows [n, dim] and table [vocab, dim] with dense features."""
    _refuse(ids.dtype.is_floating_point or ids.dtype.is_complex or ids.element_size() not in (4, 8) or not ids.is_contiguous(), "ids: a dense tensor of 4- or 8-byte integers is wanted")
    _refuse(rows.dim() != 2 or table.dim() != 2 or rows.shape[0] != ids.numel() or rows.shape[1] != table.shape[1], "one row of the table's width per token is wanted")
    _refuse((rows.stride(1) != 1 or table.stride(1) != 1) and table.shape[1] > 1, "features have to be dense")


def _row_stride(t) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def embedding(ids, weight, out, scale: float = 1.0, ws=None, stream=None) -> None:
    """out[t] = scale * weight[ids[t]]; zeros where ids[t] is negative (or not below the table's height: fault word 2 of ws)."""
    _check_tokens(ids, out, weight)
    rc = load().tcuscan_embedding(ids.data_ptr(), ids.element_size(), ids.numel(), weight.data_ptr(), weight.shape[0], weight.shape[1], _row_stride(weight),
                                  _element(weight), out.data_ptr(), _row_stride(out), _element(out), scale, *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_embedding")


def embedding_backward_workspace_bytes(n: int, vocab: int, dim: int) -> int:
    return int(load().tcuscan_embedding_backward_workspace_bytes(n, vocab, dim))


def new_embedding_backward_workspace(n: int, vocab: int, dim: int):
    """A zero-filled workspace for embedding_backward of n tokens."""
    return _zeros(embedding_backward_workspace_bytes(n, vocab, dim))


def embedding_backward(ids, d_out, d_weight, scale: float = 1.0, padding: int = -1, accumulate: bool = False, ws=None, stream=None) -> None:
    """d_weight[r] = scale * (sum of d_out[t] over the tokens t with ids[t] == r), or added to it; tokens numbered `padding` add nothing."""
    _check_tokens(ids, d_out, d_weight)
    rc = load().tcuscan_embedding_backward(ids.data_ptr(), ids.element_size(), ids.numel(), d_out.data_ptr(), _row_stride(d_out), _element(d_out),
                                           d_weight.data_ptr(), d_weight.shape[0], d_weight.shape[1], _row_stride(d_weight), _element(d_weight), scale,
                                           int(padding), ACCUMULATE if accumulate else 0, *_ws_args(ws), _stream(stream))
    if rc != OK:
        raise TcuscanError(rc, "tcuscan_embedding_backward")
