"""Thin ctypes binding of libkvr.so (declared in include/kvr.h).

Argument marshalling only: every function has the name and the argument order
of its C entry point, takes torch tensors where the C call takes device
pointers, checks dtype / device / contiguity / minimum size, and passes
`data_ptr()` plus the current torch HIP stream.  Nothing is computed here.
There is no fallback: if the library is missing, loading raises.

The calls of a decode step (`kvr_step_update`, `kvr_attend_decode`) and those over an
uncompressed cache (`kvr_rotate`, `kvr_attend_paged`, `kvr_attend_prompt`) are checked and
made by the extension `_kvr_fast` (csrc/kvr_fast.c), where it was built
and every argument is as it should be; anything else comes back to the checks here,
which raise.
"""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import os

import torch

KVR_OK = 0
KVR_ERR_INVALID_ARG = -1
KVR_ERR_UNSUPPORTED = -2
KVR_ERR_WORKSPACE_TOO_SMALL = -3
KVR_ERR_HIP = -4
KVR_F32, KVR_BF16 = 0, 1
KVR_MEDIAN_MIDMEAN, KVR_MEDIAN_LOWER = 0, 1
KVR_OP_SELECT, KVR_OP_ENCODE, KVR_OP_RECONSTRUCT, KVR_OP_ATTEND = 0, 1, 2, 3
KVR_MAX_ROWS = 8
KVR_HEAD_DIM = 128

_ERR_NAMES = {-1: "KVR_ERR_INVALID_ARG", -2: "KVR_ERR_UNSUPPORTED",
              -3: "KVR_ERR_WORKSPACE_TOO_SMALL", -4: "KVR_ERR_HIP"}

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libkvr.so")
# named for the interpreter it was built for; another one's is not looked at
FAST_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_kvr_fast" + importlib.machinery.EXTENSION_SUFFIXES[0])

EXPORTS = ["kvr_version", "kvr_last_hip_error", "kvr_recent_size", "kvr_hash_params_from_seed", "kvr_hash_host",
           "kvr_workspace_size", "kvr_append", "kvr_select", "kvr_encode", "kvr_compact", "kvr_step_update",
           "kvr_swap_back", "kvr_reconstruct", "kvr_attend_decode", "kvr_attend_decode_static",
           "kvr_attend_multi_workspace_size", "kvr_attend_multi"]
EXPORTS += ["kvr_rotate", "kvr_attend_prompt_workspace_size", "kvr_attend_prompt", "kvr_attend_paged_workspace_size",
            "kvr_attend_paged", "kvr_rotate_axes", "kvr_attend_shared_workspace_size", "kvr_attend_shared"]
KVR_MAX_AXES = 8
KVR_ROTATE_HALVES, KVR_ROTATE_PAIRS = 0, 1
KVR_STATIC_SCRATCH_BYTES = 80 << 20


class KvrError(RuntimeError):
    def __init__(self, fn, code, hip=0):
        self.code = code
        self.hip = hip
        super().__init__(f"{fn} failed: {_ERR_NAMES.get(code, code)}" + (f" (hipError {hip})" if hip else ""))


class kvr_desc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("r", C.c_int32), ("w", C.c_int32), ("dtype", C.c_int32),
                ("sign_mask", C.c_int32), ("median_mode", C.c_int32), ("softmax_scale", C.c_float),
                ("hash_params", (C.c_uint64 * 4) * KVR_MAX_ROWS)]


class kvr_attend_opts(C.Structure):
    _fields_ = [("side_stream", C.c_void_p), ("fork_event", C.c_void_p), ("join_event", C.c_void_p),
                ("prof_start", C.c_void_p), ("prof_stop", C.c_void_p)]


class kvr_pages(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("table", C.c_void_p),
                ("n_pages", C.c_int32), ("page_size", C.c_int32), ("table_cap", C.c_int32)]


class kvr_rotation(C.Structure):
    _fields_ = [("q_weight", C.c_void_p), ("k_weight", C.c_void_p), ("inv_freq", C.c_void_p),
                ("eps", C.c_float), ("rot_dim", C.c_int32), ("style", C.c_int32)]


class kvr_axes(C.Structure):
    _fields_ = [("n_axes", C.c_int32), ("axis", C.c_uint8 * (KVR_HEAD_DIM // 2))]


class kvr_groups(C.Structure):
    _fields_ = [("start", C.c_void_p), ("n_shared", C.c_void_p), ("n_groups", C.c_int32)]


_fast = None
_lib = None
_hip = None


def hip() -> C.CDLL:
    """The HIP runtime, for the few raw handles the C ABI takes (events)."""
    global _hip
    if _hip is None:
        h = C.CDLL("libamdhip64.so")
        h.hipEventCreateWithFlags.argtypes = [C.POINTER(C.c_void_p), C.c_uint]
        h.hipEventElapsedTime.argtypes = [C.POINTER(C.c_float), C.c_void_p, C.c_void_p]
        h.hipEventDestroy.argtypes = [C.c_void_p]
        _hip = h
    return _hip


def event_create(timing: bool) -> C.c_void_p:
    ev = C.c_void_p()
    rc = hip().hipEventCreateWithFlags(C.byref(ev), 0 if timing else 2)      # 2 = hipEventDisableTiming
    if rc != 0:
        raise RuntimeError(f"hipEventCreateWithFlags failed: {rc}")
    return ev


def event_elapsed_ms(a, b) -> float:
    ms = C.c_float()
    rc = hip().hipEventElapsedTime(C.byref(ms), a, b)
    if rc != 0:
        raise RuntimeError(f"hipEventElapsedTime failed: {rc}")
    return ms.value


class SideStream:
    """A second stream (default priority) and the fork / join events that a caller
    lends to kvr_attend_decode.  Used where retained slots and Vague list are separate
    kernels (bf16, a sketch that only the general staged kernel holds) and the list
    fills the chip twice over; other calls make one launch for both and leave it alone.
    Plumbing only.  One object serves any number of calls that are ordered on one
    stream."""

    def __init__(self, device="cuda"):
        self.stream = torch.cuda.Stream(device=device)
        self.fork = event_create(False)
        self.join = event_create(False)

    def opts(self, prof_start=None, prof_stop=None) -> "kvr_attend_opts":
        return kvr_attend_opts(self.stream.cuda_stream, self.fork, self.join, prof_start, prof_stop)

    def __del__(self):
        try:
            hip().hipEventDestroy(self.fork)
            hip().hipEventDestroy(self.join)
        except Exception:
            pass


def lib() -> C.CDLL:
    """Load libkvr.so (built by paper_2512_17917_amd.build); raises if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2512_17917_amd.build`")
        L = C.CDLL(LIB_PATH)
        vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
        dp = C.POINTER(kvr_desc)
        L.kvr_version.restype = C.c_char_p
        L.kvr_version.argtypes = []
        L.kvr_last_hip_error.restype = i32
        L.kvr_last_hip_error.argtypes = []
        L.kvr_recent_size.restype = i32
        L.kvr_recent_size.argtypes = [i32, i32, i32]
        L.kvr_hash_params_from_seed.restype = i32
        L.kvr_hash_params_from_seed.argtypes = [C.c_uint64, i32, C.POINTER(C.c_uint64)]
        L.kvr_hash_host.restype = i32
        L.kvr_hash_host.argtypes = [dp, i32, C.POINTER(i32), C.POINTER(i32)]
        L.kvr_workspace_size.restype = i32
        L.kvr_workspace_size.argtypes = [dp, i32, i64, i64, C.POINTER(sz)]
        L.kvr_append.restype = i32
        L.kvr_append.argtypes = [dp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
        L.kvr_select.restype = i32
        L.kvr_select.argtypes = [dp, vp, i64, vp, i32, vp, i32, i32, vp, vp, vp, i32, vp, vp, i32,
                                 vp, sz, vp]
        L.kvr_encode.restype = i32
        L.kvr_encode.argtypes = [dp, vp, vp, i32, vp, vp, vp, i32, vp, vp, vp, vp, vp, sz, vp]
        L.kvr_compact.restype = i32
        L.kvr_compact.argtypes = [dp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, i32, i32, vp]
        L.kvr_step_update.restype = i32
        L.kvr_step_update.argtypes = [dp, vp, vp, vp, vp, vp, vp, i32, vp, i64, i32, i32, vp, vp, vp, i32,
                                      vp, vp, i32, vp, vp, vp]
        L.kvr_swap_back.restype = i32
        L.kvr_swap_back.argtypes = [dp, vp, i64, vp, vp, vp, i32, vp, i32, C.c_float, i32, vp, vp, vp, vp, i32,
                                    vp, vp, vp]
        L.kvr_reconstruct.restype = i32
        L.kvr_reconstruct.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp, vp]
        L.kvr_attend_decode.restype = i32
        L.kvr_attend_decode.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, i64,
                                        vp, sz, C.POINTER(kvr_attend_opts), vp]
        L.kvr_attend_decode_static.restype = i32
        L.kvr_attend_decode_static.argtypes = [dp, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, i64,
                                               C.POINTER(kvr_attend_opts), vp]
        L.kvr_attend_multi_workspace_size.restype = i32
        L.kvr_attend_multi_workspace_size.argtypes = [dp, i32, i64, i64, C.POINTER(sz)]
        L.kvr_attend_multi.restype = i32
        L.kvr_attend_multi.argtypes = [dp, vp, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, i64,
                                       vp, sz, vp]
        pp = C.POINTER(kvr_pages)
        L.kvr_rotate.restype = i32
        L.kvr_rotate.argtypes = [dp, C.POINTER(kvr_rotation), vp, i64, vp, i64, vp, i64, i32, vp, vp, vp, vp, pp, vp]
        L.kvr_rotate_axes.restype = i32
        L.kvr_rotate_axes.argtypes = [dp, C.POINTER(kvr_rotation), C.POINTER(kvr_axes), vp, i64, vp, i64, vp, i64, vp, i64, i32,
                                      vp, vp, vp, vp, pp, vp]
        L.kvr_attend_prompt_workspace_size.restype = i32
        L.kvr_attend_prompt_workspace_size.argtypes = [dp, i32, pp, i32, i32, i32, C.POINTER(sz)]
        L.kvr_attend_prompt.restype = i32
        L.kvr_attend_prompt.argtypes = [dp, vp, i32, vp, vp, pp, i32, i32, vp, vp, i64, vp, sz, vp]
        L.kvr_attend_paged_workspace_size.restype = i32
        L.kvr_attend_paged_workspace_size.argtypes = [dp, pp, i32, i32, i32, C.POINTER(sz)]
        L.kvr_attend_paged.restype = i32
        L.kvr_attend_paged.argtypes = [dp, vp, vp, pp, i32, i32, vp, vp, i64, vp, sz, vp]
        gp = C.POINTER(kvr_groups)
        L.kvr_attend_shared_workspace_size.restype = i32
        L.kvr_attend_shared_workspace_size.argtypes = [dp, i32, pp, gp, i32, i32, i32, C.POINTER(sz)]
        L.kvr_attend_shared.restype = i32
        L.kvr_attend_shared.argtypes = [dp, vp, i32, vp, vp, pp, gp, i32, i32, vp, vp, i64, vp, sz, vp]
        _load_fast(L)
        _lib = L
    return _lib


def _load_fast(L):
    """The calls of a decode step make some thirty tensor checks, 0.75 us each in Python; _kvr_fast makes the same
    checks in C and hands back None where one fails, so that the Python code below says what is wrong."""
    global _fast
    if os.path.exists(FAST_PATH):
        spec = importlib.util.spec_from_file_location("_kvr_fast", FAST_PATH)
        m = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(m)
        address = lambda f: C.cast(f, C.c_void_p).value
        m.setup(address(L.kvr_step_update), address(L.kvr_attend_decode), torch.float32, torch.bfloat16, torch.int32,
                torch.uint8, torch.Tensor)
        m.setup_cache(address(L.kvr_rotate), address(L.kvr_attend_paged), address(L.kvr_attend_prompt))
        m.setup_more(address(L.kvr_rotate_axes), address(L.kvr_attend_shared))
        _fast = m


def _check(fn, rc):
    if rc != KVR_OK:
        raise KvrError(fn, rc, lib().kvr_last_hip_error() if rc == KVR_ERR_HIP else 0)


def make_desc(batch, n_q_heads, n_kv_heads, r, w, dtype, *, seed=None, hash_params=None,
              sign_mask=2, median_mode=KVR_MEDIAN_MIDMEAN, softmax_scale=None, head_dim=KVR_HEAD_DIM):
    """Fill a kvr_desc.  dtype: torch.float32 / torch.bfloat16 or KVR_F32 / KVR_BF16.
    hash_params: r rows of (a, b, c, d), or derived from `seed` by the library."""
    d = kvr_desc()
    d.batch, d.n_q_heads, d.n_kv_heads, d.head_dim = batch, n_q_heads, n_kv_heads, head_dim
    d.r, d.w = r, w
    if dtype in (torch.float32, KVR_F32):
        d.dtype = KVR_F32
    elif dtype in (torch.bfloat16, KVR_BF16):
        d.dtype = KVR_BF16
    else:
        raise ValueError(f"unsupported dtype {dtype}")
    d.sign_mask, d.median_mode = sign_mask, median_mode
    d.softmax_scale = (head_dim ** -0.5) if softmax_scale is None else softmax_scale
    if hash_params is None:
        hash_params = kvr_hash_params_from_seed(0 if seed is None else seed, r)
    for i, row in enumerate(hash_params):
        for k in range(4):
            d.hash_params[i][k] = int(row[k]) & ((1 << 64) - 1)
    return d


def desc_hash_params(d: kvr_desc):
    return [tuple(int(d.hash_params[i][k]) for k in range(4)) for i in range(d.r)]


def _torch_dtype(d: kvr_desc):
    return torch.float32 if d.dtype == KVR_F32 else torch.bfloat16


def _ptr(t, dtype, min_numel, name, allow_none=False):
    if t is None:
        if allow_none:
            return None
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() < min_numel:
        raise ValueError(f"{name}: {t.numel()} elements, need at least {min_numel}")
    return t.data_ptr()


def _stream():
    return torch.cuda.current_stream().cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_of(dev):
    """_stream() of the current device, whose index the caller has (2.7 us less where torch offers the bare handle)."""
    return _raw_stream(dev) if _raw_stream is not None else _stream()


def _ws(ws):
    if ws is None:
        return None, 0
    if not (isinstance(ws, torch.Tensor) and ws.is_cuda and ws.is_contiguous()):
        raise ValueError("ws must be a contiguous device tensor")
    return ws.data_ptr(), ws.numel() * ws.element_size()


# ---------------------------------------------------------------------------
def kvr_version() -> str:
    return lib().kvr_version().decode()


def kvr_recent_size(r_size: int, r_budget: int, slack: int) -> int:
    rc = lib().kvr_recent_size(r_size, r_budget, slack)
    if rc < 0:
        raise KvrError("kvr_recent_size", rc)
    return int(rc)


def kvr_hash_params_from_seed(seed: int, r: int):
    buf = (C.c_uint64 * (4 * r))()
    _check("kvr_hash_params_from_seed", lib().kvr_hash_params_from_seed(seed & ((1 << 64) - 1), r, buf))
    return [tuple(int(buf[i * 4 + k]) for k in range(4)) for i in range(r)]


def kvr_hash_host(desc: kvr_desc, J: int):
    b = (C.c_int32 * KVR_MAX_ROWS)()
    s = (C.c_int32 * KVR_MAX_ROWS)()
    _check("kvr_hash_host", lib().kvr_hash_host(C.byref(desc), J, b, s))
    return [int(b[i]) for i in range(desc.r)], [int(s[i]) for i in range(desc.r)]


def kvr_workspace_size(desc: kvr_desc, op: int, n_a: int, n_b: int = 0) -> int:
    out = C.c_size_t(0)
    _check("kvr_workspace_size", lib().kvr_workspace_size(C.byref(desc), op, n_a, n_b, C.byref(out)))
    return int(out.value)


def alloc_workspace(desc: kvr_desc, op: int, n_a: int, n_b: int = 0, device="cuda") -> torch.Tensor:
    n = kvr_workspace_size(desc, op, n_a, n_b)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def kvr_append(desc, k_new, v_new, n_ctx, k_ret, v_ret, ret_pos, ret_cap, out_slot=None):
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    rc = lib().kvr_append(
        C.byref(desc), _ptr(k_new, dt, U * D, "k_new"), _ptr(v_new, dt, U * D, "v_new"),
        _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"),
        _ptr(k_ret, dt, U * ret_cap * D, "k_ret"), _ptr(v_ret, dt, U * ret_cap * D, "v_ret"),
        _ptr(ret_pos, torch.int32, U * ret_cap, "ret_pos"), ret_cap,
        _ptr(out_slot, torch.int32, U, "out_slot", True), _stream())
    _check("kvr_append", rc)


def kvr_select(desc, scores, n_cap, ret_pos, ret_cap, n_ctx, n_recent, k_candidate,
               evict_slot, evict_pos, n_evict, evict_cap, vague_pos, n_vague, vague_cap, ws=None):
    U = desc.batch * desc.n_kv_heads
    wp, wb = _ws(ws)
    rc = lib().kvr_select(
        C.byref(desc), _ptr(scores, torch.float32, U * n_cap, "scores"), n_cap,
        _ptr(ret_pos, torch.int32, U * ret_cap, "ret_pos"), ret_cap,
        _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"), n_recent, k_candidate,
        _ptr(evict_slot, torch.int32, U * evict_cap, "evict_slot"),
        _ptr(evict_pos, torch.int32, U * evict_cap, "evict_pos"),
        _ptr(n_evict, torch.int32, U, "n_evict"), evict_cap,
        _ptr(vague_pos, torch.int32, U * vague_cap, "vague_pos", True),
        _ptr(n_vague, torch.int32, U, "n_vague", True), vague_cap, wp, wb, _stream())
    _check("kvr_select", rc)


def kvr_encode(desc, k_src, v_src, src_rows, src_slot, tok_pos, count, cap, sketch_k, sketch_v,
               out_bucket=None, out_sign=None, ws=None):
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    S = desc.r * desc.w * D
    wp, wb = _ws(ws)
    rc = lib().kvr_encode(
        C.byref(desc), _ptr(k_src, dt, U * src_rows * D, "k_src"), _ptr(v_src, dt, U * src_rows * D, "v_src"),
        src_rows, _ptr(src_slot, torch.int32, U * cap, "src_slot"),
        _ptr(tok_pos, torch.int32, U * cap, "tok_pos"), _ptr(count, torch.int32, U, "count"), cap,
        _ptr(sketch_k, dt, U * S, "sketch_k"), _ptr(sketch_v, dt, U * S, "sketch_v"),
        _ptr(out_bucket, torch.int32, U * cap * desc.r, "out_bucket", True),
        _ptr(out_sign, torch.uint8, U * cap, "out_sign", True), wp, wb, _stream())
    _check("kvr_encode", rc)


def kvr_compact(desc, k_src, v_src, src_pos, src_cap, evict_slot, n_evict, evict_cap, k_ret, v_ret, ret_pos, ret_cap,
                max_keep):
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    rc = lib().kvr_compact(
        C.byref(desc), _ptr(k_src, dt, U * src_cap * D, "k_src"), _ptr(v_src, dt, U * src_cap * D, "v_src"),
        _ptr(src_pos, torch.int32, U * src_cap, "src_pos"), src_cap,
        _ptr(evict_slot, torch.int32, U * evict_cap, "evict_slot"), _ptr(n_evict, torch.int32, U, "n_evict"), evict_cap,
        _ptr(k_ret, dt, U * ret_cap * D, "k_ret"), _ptr(v_ret, dt, U * ret_cap * D, "v_ret"),
        _ptr(ret_pos, torch.int32, U * ret_cap, "ret_pos"), ret_cap, max_keep, _stream())
    _check("kvr_compact", rc)


def kvr_step_update(desc, k_new, v_new, n_ctx, k_ret, v_ret, ret_pos, ret_cap, scores, n_cap, n_recent,
                    k_candidate, evict_slot, evict_pos, n_evict, evict_cap, vague_pos, n_vague, vague_cap,
                    sketch_k, sketch_v):
    lib()
    if _fast is not None and isinstance(desc, kvr_desc) and isinstance(k_new, torch.Tensor) and k_new.is_cuda:
        rc = _fast.step_update(C.addressof(desc), _stream(), k_new, v_new, n_ctx, k_ret, v_ret, ret_pos, ret_cap, scores, n_cap,
                               n_recent, k_candidate, evict_slot, evict_pos, n_evict, evict_cap, vague_pos, n_vague, vague_cap,
                               sketch_k, sketch_v)
        if rc is not None:
            return _check("kvr_step_update", rc)
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    S = desc.r * desc.w * D
    rc = lib().kvr_step_update(
        C.byref(desc), _ptr(k_new, dt, U * D, "k_new"), _ptr(v_new, dt, U * D, "v_new"),
        _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"),
        _ptr(k_ret, dt, U * ret_cap * D, "k_ret"), _ptr(v_ret, dt, U * ret_cap * D, "v_ret"),
        _ptr(ret_pos, torch.int32, U * ret_cap, "ret_pos"), ret_cap,
        _ptr(scores, torch.float32, U * n_cap, "scores"), n_cap, n_recent, k_candidate,
        _ptr(evict_slot, torch.int32, U * evict_cap, "evict_slot"),
        _ptr(evict_pos, torch.int32, U * evict_cap, "evict_pos"),
        _ptr(n_evict, torch.int32, U, "n_evict"), evict_cap,
        _ptr(vague_pos, torch.int32, U * vague_cap, "vague_pos", True),
        _ptr(n_vague, torch.int32, U, "n_vague", True), vague_cap,
        _ptr(sketch_k, dt, U * S, "sketch_k"), _ptr(sketch_v, dt, U * S, "sketch_v"), _stream())
    _check("kvr_step_update", rc)


def kvr_swap_back(desc, scores, n_cap, k_ret, v_ret, ret_pos, ret_cap, n_ctx, n_recent, replace_rate,
                  max_swaps, sketch_k, sketch_v, vague_pos, n_vague, vague_cap, n_swapped=None, swap_log=None):
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    S = desc.r * desc.w * D
    rc = lib().kvr_swap_back(
        C.byref(desc), _ptr(scores, torch.float32, U * n_cap, "scores"), n_cap,
        _ptr(k_ret, dt, U * ret_cap * D, "k_ret"), _ptr(v_ret, dt, U * ret_cap * D, "v_ret"),
        _ptr(ret_pos, torch.int32, U * ret_cap, "ret_pos"), ret_cap,
        _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"), n_recent, C.c_float(replace_rate), max_swaps,
        _ptr(sketch_k, dt, U * S, "sketch_k"), _ptr(sketch_v, dt, U * S, "sketch_v"),
        _ptr(vague_pos, torch.int32, U * vague_cap, "vague_pos"), _ptr(n_vague, torch.int32, U, "n_vague"),
        vague_cap, _ptr(n_swapped, torch.int32, U, "n_swapped", True),
        _ptr(swap_log, torch.int32, U * max(max_swaps, 1) * 2, "swap_log", True), _stream())
    _check("kvr_swap_back", rc)


def kvr_reconstruct(desc, sketch_k, sketch_v, tok_pos, count, cap, k_out, v_out):
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    S = desc.r * desc.w * D
    rc = lib().kvr_reconstruct(
        C.byref(desc), _ptr(sketch_k, dt, U * S, "sketch_k"), _ptr(sketch_v, dt, U * S, "sketch_v"),
        _ptr(tok_pos, torch.int32, U * cap, "tok_pos"), _ptr(count, torch.int32, U, "count"), cap,
        _ptr(k_out, dt, U * cap * D, "k_out"), _ptr(v_out, dt, U * cap * D, "v_out"), _stream())
    _check("kvr_reconstruct", rc)


def kvr_attend_decode(desc, q, k_ret, v_ret, ret_pos, ret_cap, sketch_k, sketch_v, vague_pos, n_vague,
                      vague_cap, out, scores, n_cap, ws, opts=None):
    lib()
    if (_fast is not None and isinstance(desc, kvr_desc) and (opts is None or isinstance(opts, kvr_attend_opts))
            and isinstance(q, torch.Tensor) and q.is_cuda):
        rc = _fast.attend_decode(C.addressof(desc), _stream(), C.addressof(opts) if opts is not None else 0, q, k_ret, v_ret,
                                 ret_pos, ret_cap, sketch_k, sketch_v, vague_pos, n_vague, vague_cap, out, scores, n_cap, ws)
        if rc is not None:
            return _check("kvr_attend_decode", rc)
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    S = desc.r * desc.w * D
    wp, wb = _ws(ws)
    rc = lib().kvr_attend_decode(
        C.byref(desc), _ptr(q, dt, desc.batch * desc.n_q_heads * D, "q"),
        _ptr(k_ret, dt, U * ret_cap * D, "k_ret"), _ptr(v_ret, dt, U * ret_cap * D, "v_ret"),
        _ptr(ret_pos, torch.int32, U * ret_cap, "ret_pos", True), ret_cap,
        _ptr(sketch_k, dt, U * S, "sketch_k", True), _ptr(sketch_v, dt, U * S, "sketch_v", True),
        _ptr(vague_pos, torch.int32, U * vague_cap, "vague_pos", True),
        _ptr(n_vague, torch.int32, U, "n_vague", True), vague_cap,
        _ptr(out, torch.float32, desc.batch * desc.n_q_heads * D, "out"),
        _ptr(scores, torch.float32, U * n_cap, "scores", True), n_cap, wp, wb,
        C.byref(opts) if opts is not None else None, _stream())
    _check("kvr_attend_decode", rc)


def kvr_attend_decode_static(desc, q, k_ret, v_ret, ret_pos, ret_cap, sketch_k, sketch_v, vague_pos, n_vague,
                             vague_cap, out, scores, n_cap, opts=None):
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    S = desc.r * desc.w * D
    rc = lib().kvr_attend_decode_static(
        C.byref(desc), _ptr(q, dt, desc.batch * desc.n_q_heads * D, "q"),
        _ptr(k_ret, dt, U * ret_cap * D, "k_ret"), _ptr(v_ret, dt, U * ret_cap * D, "v_ret"),
        _ptr(ret_pos, torch.int32, U * ret_cap, "ret_pos", True), ret_cap,
        _ptr(sketch_k, dt, U * S, "sketch_k", True), _ptr(sketch_v, dt, U * S, "sketch_v", True),
        _ptr(vague_pos, torch.int32, U * vague_cap, "vague_pos", True),
        _ptr(n_vague, torch.int32, U, "n_vague", True), vague_cap,
        _ptr(out, torch.float32, desc.batch * desc.n_q_heads * D, "out"),
        _ptr(scores, torch.float32, U * n_cap, "scores", True), n_cap,
        C.byref(opts) if opts is not None else None, _stream())
    _check("kvr_attend_decode_static", rc)


def kvr_attend_multi_workspace_size(desc, n_q, ret_cap, vague_cap) -> int:
    n = C.c_size_t(0)
    _check("kvr_attend_multi_workspace_size",
           lib().kvr_attend_multi_workspace_size(C.byref(desc), n_q, ret_cap, vague_cap, C.byref(n)))
    return n.value


def kvr_attend_multi(desc, q, n_q, n_ctx, k_ret, v_ret, ret_pos, ret_cap, sketch_k, sketch_v, vague_pos, n_vague,
                     vague_cap, out, scores, n_cap, ws):
    U, D, dt = desc.batch * desc.n_kv_heads, desc.head_dim, _torch_dtype(desc)
    S = desc.r * desc.w * D
    wp, wb = _ws(ws)
    rc = lib().kvr_attend_multi(
        C.byref(desc), _ptr(q, dt, desc.batch * n_q * desc.n_q_heads * D, "q"), n_q,
        _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"),
        _ptr(k_ret, dt, U * ret_cap * D, "k_ret"), _ptr(v_ret, dt, U * ret_cap * D, "v_ret"),
        _ptr(ret_pos, torch.int32, U * ret_cap, "ret_pos"), ret_cap,
        _ptr(sketch_k, dt, U * S, "sketch_k", True), _ptr(sketch_v, dt, U * S, "sketch_v", True),
        _ptr(vague_pos, torch.int32, U * vague_cap, "vague_pos", True),
        _ptr(n_vague, torch.int32, U, "n_vague", True), vague_cap,
        _ptr(out, torch.float32, desc.batch * n_q * desc.n_q_heads * D, "out"),
        _ptr(scores, torch.float32, U * n_cap, "scores", True), n_cap, wp, wb, _stream())
    _check("kvr_attend_multi", rc)


# ---------------------------------------------------------------------------
# the uncompressed cache
def _here(*tensors):
    """The tensors of a call live on the current device, whose stream it is enqueued on."""
    there = [t.device for t in tensors if isinstance(t, torch.Tensor) and t.is_cuda]
    if there and any(x.index != torch.cuda.current_device() for x in there):
        raise ValueError(f"tensors live on {sorted(set(map(str, there)))}, the current device is "
                         f"cuda:{torch.cuda.current_device()}")


def _one_device(*tensors):
    """Index of the device that the tensors share, None if there are none."""
    there = {t.device.index for t in tensors if t is not None}
    if len(there) > 1:
        raise ValueError("the tensors live on different devices")
    return there.pop() if there else None


def make_pages(desc, k, v, table=None):
    """kvr_pages over the pools k, v [n_pages, Hkv, page_size, D] and table int32 [B, table_cap]; without a table the
    pools are a dense cache [B, Hkv, tokens, D].  The struct keeps the tensors."""
    dt = _torch_dtype(desc)
    for t, name in ((k, "k"), (v, "v")):
        if not isinstance(t, torch.Tensor) or t.dim() != 4:
            raise ValueError(f"{name} must be a tensor [n_pages, n_kv_heads, page_size, head_dim]")
        if tuple(t.shape) != tuple(k.shape) or t.shape[1] != desc.n_kv_heads or t.shape[3] != desc.head_dim:
            raise ValueError(f"{name}: shape {tuple(t.shape)} does not fit the descriptor or the other pool")
    p = kvr_pages(_ptr(k, dt, 1, "k"), _ptr(v, dt, 1, "v"), None, k.shape[0], k.shape[2], 0)
    if table is not None:
        if not isinstance(table, torch.Tensor) or table.dim() != 2 or table.shape[0] < desc.batch:
            raise ValueError("table must be a tensor [batch, table_cap]")
        p.table, p.table_cap = _ptr(table, torch.int32, 1, "table"), table.shape[1]
    p.tensors = (k, v, table)
    p.fits = (desc.dtype, desc.n_kv_heads, desc.head_dim, k.shape[0] if table is None else table.shape[0])
    p.dev = _one_device(k, v, table)
    return p


def _pages(desc, p, allow_none=False):
    """A kvr_pages of make_pages that fits this descriptor (it may have been made with another one)."""
    if p is None and allow_none:
        return None
    if not isinstance(p, kvr_pages) or not hasattr(p, "fits"):
        raise TypeError("pages must come from make_pages")
    dtype, heads, dim, rows = p.fits
    if dtype != desc.dtype or heads != desc.n_kv_heads or dim != desc.head_dim or rows < desc.batch:
        raise ValueError("pages were made for another kind of descriptor")
    if p.dev != torch.cuda.current_device():
        raise ValueError(f"the pages live on cuda:{p.dev}, the current device is cuda:{torch.cuda.current_device()}")
    return C.byref(p)


def make_rotation(desc, inv_freq=None, *, q_weight=None, k_weight=None, eps=1e-6, pairs=False):
    """kvr_rotation: inv_freq float64 [rot_dim / 2] (None: nothing is turned), weights [D] of the norms (None: no norm),
    pairs: channels 2i and 2i + 1 make a pair instead of i and i + rot_dim / 2.  The struct keeps the tensors."""
    dt = _torch_dtype(desc)
    n = 0 if inv_freq is None else inv_freq.numel()
    r = kvr_rotation(_ptr(q_weight, dt, desc.head_dim, "q_weight", True), _ptr(k_weight, dt, desc.head_dim, "k_weight", True),
                     _ptr(inv_freq, torch.float64, 1, "inv_freq") if n else None, eps, 2 * n,
                     KVR_ROTATE_PAIRS if pairs else KVR_ROTATE_HALVES)
    r.tensors = (inv_freq, q_weight, k_weight)
    r.weights = None if q_weight is None and k_weight is None else desc.dtype
    r.dev = _one_device(*r.tensors)
    return r


def _rows(t, dtype, n_rows, heads, d, name):
    """Pointer and row stride of [n_rows, heads, D] with dense heads and rows any way apart."""
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    if t.dim() != 3 or t.shape[0] < n_rows or t.shape[1] != heads or t.shape[2] != d:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, need [{n_rows}, {heads}, {d}]")
    if t.stride(2) != 1 or (heads > 1 and t.stride(1) != d):
        raise ValueError(f"{name}: the heads of a row must be dense")
    return t.data_ptr(), t.stride(0) if n_rows > 1 else heads * d


def _rotation(desc, rot):
    if not isinstance(rot, kvr_rotation) or not hasattr(rot, "tensors"):
        raise TypeError("rot must come from make_rotation")
    if rot.weights is not None and rot.weights != desc.dtype:
        raise ValueError("the rotation's weights were made for another kind of descriptor")


def kvr_rotate(desc, rot, q, k, v, n_rows, q_start, n_ctx, q_out, k_out=None, pages=None):
    """As the C call; the rows' strides are the tensors' own."""
    _rotation(desc, rot)
    pp = _pages(desc, pages, True)
    lib()
    one = q if q is not None else k
    if _fast is not None and isinstance(desc, kvr_desc) and isinstance(one, torch.Tensor) and one.is_cuda:
        dev = torch.cuda.current_device()
        if rot.dev is not None and rot.dev != dev:
            raise ValueError(f"the rotation lives on cuda:{rot.dev}, the current device is cuda:{dev}")
        rc = _fast.rotate(C.addressof(desc), C.addressof(rot), C.addressof(pages) if pages is not None else 0, dev,
                          _stream_of(dev), q, k, v, n_rows, q_start, n_ctx, q_out, k_out)
        if rc is not None:
            return _check("kvr_rotate", rc)
    dt, d = _torch_dtype(desc), desc.head_dim
    qp, qs = _rows(q, dt, n_rows, desc.n_q_heads, d, "q")
    kp, ks = _rows(k, dt, n_rows, desc.n_kv_heads, d, "k")
    vp, vs = _rows(v, dt, n_rows, desc.n_kv_heads, d, "v")
    _here(q, k, v, q_start, n_ctx, q_out, k_out, *rot.tensors)
    rc = lib().kvr_rotate(
        C.byref(desc), C.byref(rot), qp, qs, kp, ks, vp, vs, n_rows,
        _ptr(q_start, torch.int32, desc.batch + 1, "q_start", True), _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"),
        _ptr(q_out, dt, n_rows * desc.n_q_heads * d, "q_out", True),
        _ptr(k_out, dt, n_rows * desc.n_kv_heads * d, "k_out", True), pp, _stream())
    _check("kvr_rotate", rc)


def make_axes(axis, n_axes=None):
    """kvr_axes: the axis of each turned pair of channels, as many as the rotation has; n_axes: how many axes there are
    (None: the largest of them and those before it)."""
    axis = [int(x) for x in axis]
    n = max(axis, default=0) + 1 if n_axes is None else int(n_axes)
    if not 1 <= n <= KVR_MAX_AXES or len(axis) > KVR_HEAD_DIM // 2 or any(not 0 <= x < n for x in axis):
        raise ValueError(f"axes: {len(axis)} pairs of at most {KVR_HEAD_DIM // 2}, axes 0 .. {n - 1} of at most {KVR_MAX_AXES}")
    a = kvr_axes(n, (C.c_uint8 * (KVR_HEAD_DIM // 2))(*axis))
    a.pairs = len(axis)
    return a


def kvr_rotate_axes(desc, rot, axes, pos, q, k, v, n_rows, q_start, n_ctx, q_out, k_out=None, pages=None):
    """As the C call; the rows' strides are the tensors' own.  pos int32 [n_axes, n_rows or more], the rows of an axis dense."""
    _rotation(desc, rot)
    if not isinstance(axes, kvr_axes) or not hasattr(axes, "pairs"):
        raise TypeError("axes must come from make_axes")
    if axes.pairs != rot.rot_dim // 2:
        raise ValueError(f"axes of {axes.pairs} pairs, the rotation turns {rot.rot_dim // 2}")
    pp = _pages(desc, pages, True)
    lib()
    one = q if q is not None else k
    if _fast is not None and isinstance(desc, kvr_desc) and isinstance(one, torch.Tensor) and one.is_cuda:
        dev = torch.cuda.current_device()
        if rot.dev is not None and rot.dev != dev:
            raise ValueError(f"the rotation lives on cuda:{rot.dev}, the current device is cuda:{dev}")
        rc = _fast.rotate_axes(C.addressof(desc), C.addressof(rot), C.addressof(pages) if pages is not None else 0, dev,
                               _stream_of(dev), q, k, v, n_rows, q_start, n_ctx, q_out, k_out, C.addressof(axes), pos)
        if rc is not None:
            return _check("kvr_rotate_axes", rc)
    dt, d = _torch_dtype(desc), desc.head_dim
    qp, qs = _rows(q, dt, n_rows, desc.n_q_heads, d, "q")
    kp, ks = _rows(k, dt, n_rows, desc.n_kv_heads, d, "k")
    vp, vs = _rows(v, dt, n_rows, desc.n_kv_heads, d, "v")
    if pos is None and rot.rot_dim:
        raise ValueError("pos is required")
    if pos is not None:
        if not isinstance(pos, torch.Tensor) or pos.dtype != torch.int32:
            raise TypeError("pos must be an int32 tensor")
        if not pos.is_cuda:
            raise ValueError("pos must live in device memory")
        if pos.dim() != 2 or pos.shape[0] < axes.n_axes or pos.shape[1] < n_rows or (pos.stride(1) != 1 and pos.shape[1] > 1):
            raise ValueError(f"pos: shape {tuple(pos.shape)}, need [{axes.n_axes}, {n_rows}] with dense rows")
    _here(q, k, v, q_start, n_ctx, q_out, k_out, pos, *rot.tensors)
    rc = lib().kvr_rotate_axes(
        C.byref(desc), C.byref(rot), C.byref(axes), pos.data_ptr() if pos is not None else None,
        pos.stride(0) if pos is not None else 0, qp, qs, kp, ks, vp, vs, n_rows,
        _ptr(q_start, torch.int32, desc.batch + 1, "q_start", True),
        _ptr(n_ctx, torch.int32, desc.batch, "n_ctx", pages is None),
        _ptr(q_out, dt, n_rows * desc.n_q_heads * d, "q_out", True),
        _ptr(k_out, dt, n_rows * desc.n_kv_heads * d, "k_out", True), pp, _stream())
    _check("kvr_rotate_axes", rc)


def kvr_attend_prompt_workspace_size(desc, n_rows, pages, window, n_sink, scores) -> int:
    n = C.c_size_t(0)
    _check("kvr_attend_prompt_workspace_size", lib().kvr_attend_prompt_workspace_size(
        C.byref(desc), n_rows, _pages(desc, pages), window, n_sink, int(bool(scores)), C.byref(n)))
    return n.value


def kvr_attend_prompt(desc, q, n_rows, q_start, n_ctx, pages, window, n_sink, out, scores, n_cap, ws):
    pp = _pages(desc, pages)
    lib()
    if _fast is not None and isinstance(desc, kvr_desc) and isinstance(q, torch.Tensor) and q.is_cuda:
        dev = pages.dev                              # the current one, as _pages has found
        rc = _fast.attend_prompt(C.addressof(desc), C.addressof(pages), dev, _stream_of(dev), q, n_rows, q_start, n_ctx, window,
                                 n_sink, out, scores, n_cap, ws)
        if rc is not None:
            return _check("kvr_attend_prompt", rc)
    U, dt = desc.batch * desc.n_kv_heads, _torch_dtype(desc)
    row = desc.n_q_heads * desc.head_dim
    wp, wb = _ws(ws)
    _here(q, q_start, n_ctx, out, scores, ws)
    rc = lib().kvr_attend_prompt(
        C.byref(desc), _ptr(q, dt, n_rows * row, "q"), n_rows,
        _ptr(q_start, torch.int32, desc.batch + 1, "q_start", True), _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"),
        pp, window, n_sink, _ptr(out, dt, n_rows * row, "out"),
        _ptr(scores, torch.float32, U * n_cap, "scores", True), n_cap, wp, wb, _stream())
    _check("kvr_attend_prompt", rc)


def kvr_attend_paged_workspace_size(desc, pages, window, n_sink, scores) -> int:
    n = C.c_size_t(0)
    _check("kvr_attend_paged_workspace_size", lib().kvr_attend_paged_workspace_size(
        C.byref(desc), _pages(desc, pages), window, n_sink, int(bool(scores)), C.byref(n)))
    return n.value


def kvr_attend_paged(desc, q, n_ctx, pages, window, n_sink, out, scores, n_cap, ws):
    pp = _pages(desc, pages)
    lib()
    if _fast is not None and isinstance(desc, kvr_desc) and isinstance(q, torch.Tensor) and q.is_cuda:
        dev = pages.dev                              # the current one, as _pages has found
        rc = _fast.attend_paged(C.addressof(desc), C.addressof(pages), dev, _stream_of(dev), q, n_ctx, window,
                                n_sink, out, scores, n_cap, ws)
        if rc is not None:
            return _check("kvr_attend_paged", rc)
    U, dt = desc.batch * desc.n_kv_heads, _torch_dtype(desc)
    row = desc.batch * desc.n_q_heads * desc.head_dim
    wp, wb = _ws(ws)
    _here(q, n_ctx, out, scores, ws)
    rc = lib().kvr_attend_paged(
        C.byref(desc), _ptr(q, dt, row, "q"), _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"), pp,
        window, n_sink, _ptr(out, dt, row, "out"), _ptr(scores, torch.float32, U * n_cap, "scores", True), n_cap,
        wp, wb, _stream())
    _check("kvr_attend_paged", rc)


def make_groups(start, n_shared):
    """kvr_groups: sequences start[g] .. start[g + 1] - 1 have their first n_shared[g] tokens in common (int32 device tensors
    [n_groups + 1] and [n_groups]).  The struct keeps the tensors, whose contents may change from call to call."""
    n = n_shared.numel() if isinstance(n_shared, torch.Tensor) else 0
    g = kvr_groups(_ptr(start, torch.int32, n + 1, "start"), _ptr(n_shared, torch.int32, 0, "n_shared"), n)
    g.tensors = (start, n_shared)
    g.dev = _one_device(start, n_shared)
    return g


def _groups(groups):
    if groups is None:
        return None
    if not isinstance(groups, kvr_groups) or not hasattr(groups, "tensors"):
        raise TypeError("groups must come from make_groups")
    if groups.dev != torch.cuda.current_device():
        raise ValueError(f"the groups live on cuda:{groups.dev}, the current device is cuda:{torch.cuda.current_device()}")
    return C.byref(groups)


def kvr_attend_shared_workspace_size(desc, n_rows, pages, groups, window, n_sink, scores) -> int:
    n = C.c_size_t(0)
    _check("kvr_attend_shared_workspace_size", lib().kvr_attend_shared_workspace_size(
        C.byref(desc), n_rows, _pages(desc, pages), _groups(groups), window, n_sink, int(bool(scores)), C.byref(n)))
    return n.value


def kvr_attend_shared(desc, q, n_rows, q_start, n_ctx, pages, groups, window, n_sink, out, scores, n_cap, ws):
    pp, gp = _pages(desc, pages), _groups(groups)
    lib()
    if _fast is not None and isinstance(desc, kvr_desc) and isinstance(q, torch.Tensor) and q.is_cuda:
        dev = pages.dev                              # the current one, as _pages has found
        rc = _fast.attend_shared(C.addressof(desc), C.addressof(pages), dev, _stream_of(dev), q, n_rows, q_start, n_ctx, window,
                                 n_sink, out, scores, n_cap, ws, C.addressof(groups) if groups is not None else 0)
        if rc is not None:
            return _check("kvr_attend_shared", rc)
    U, dt = desc.batch * desc.n_kv_heads, _torch_dtype(desc)
    row = desc.n_q_heads * desc.head_dim
    wp, wb = _ws(ws)
    _here(q, q_start, n_ctx, out, scores, ws)
    rc = lib().kvr_attend_shared(
        C.byref(desc), _ptr(q, dt, n_rows * row, "q"), n_rows,
        _ptr(q_start, torch.int32, desc.batch + 1, "q_start", True), _ptr(n_ctx, torch.int32, desc.batch, "n_ctx"),
        pp, gp, window, n_sink, _ptr(out, dt, n_rows * row, "out"),
        _ptr(scores, torch.float32, U * n_cap, "scores", True), n_cap, wp, wb, _stream())
    _check("kvr_attend_shared", rc)
