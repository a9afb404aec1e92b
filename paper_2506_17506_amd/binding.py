"""ctypes binding of libvl.so.  Argument marshalling only: every step of the
path runs in the library's kernels.  torch supplies device memory and streams.

The functions carry the names of the C entry points (include/vl.h).  Handles
are returned as opaque ctypes pointers; the caller destroys them.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libvl.so")

VL_DENSE_POINTS = 1
RESULT_DTYPE = np.dtype([("status", "<u4"), ("where", "<u4"), ("a", "<u4"), ("b", "<u4")])
SUMMARY_DTYPE = np.dtype([("first_ok", "<u4"), ("passed", "<u4"), ("hist", "<u4", (4,))])                       # vl_summary
LOOP_DTYPE = np.dtype([("n_passed", "<u4"), ("max_tries", "<u4"), ("sum_tries", "<u8"), ("hist", "<u8", (4,))])  # vl_loop_stats


class VlError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {vl_strerror(code)} (code {code}, hip {vl_last_hip_error()})")
        self.code = code


class _Desc(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in
                ("n_instr", "n_vreg", "n_block", "n_occ", "n_class", "n_edge")] + \
               [(n, C.c_void_p) for n in
                ("blk_start", "succ_off", "succ", "instr_occ_off", "occ_vreg", "occ_flags",
                 "vreg_class", "vreg_width", "vreg_align", "class_size", "class_reserved")]


class _View(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in
                ("n_instr", "n_vreg", "n_block", "n_occ", "words", "n_seg", "n_tile", "tile_len",
                 "plan_len", "sweeps")] + \
               [(n, C.c_void_p) for n in
                ("live_in", "live_out", "live_after", "occ_kill", "seg_off", "seg", "hull")]


class _LanesView(C.Structure):
    _fields_ = [(n, C.c_uint32) for n in ("n_occ", "n_vreg", "n_occ_low", "n_vreg_low")] + \
               [(n, C.c_void_p) for n in ("occ_src", "occ_add", "val_vreg", "val_lane")]


class _CountJob(C.Structure):
    _fields_ = [("mir", C.c_void_p), ("live", C.c_void_p), ("cand", C.c_void_p), ("K", C.c_uint32),
                ("ld", C.c_uint64), ("out", C.c_void_p)]


class _MaskQuery(C.Structure):
    _fields_ = [("mir", C.c_void_p), ("live", C.c_void_p), ("cand", C.c_void_p), ("occ", C.c_uint32),
                ("reserved0", C.c_uint32)]


class _Job(C.Structure):
    _fields_ = [("mir", C.c_void_p), ("live", C.c_void_p), ("cand", C.c_void_p), ("K", C.c_uint32),
                ("ld", C.c_uint64), ("out", C.c_void_p)]


class _TokenRows(C.Structure):
    _fields_ = [("logits", C.c_void_p), ("ld", C.c_uint64), ("mask", C.c_void_p), ("mask_ld", C.c_uint64), ("token", C.c_void_p),
                ("n_row", C.c_uint32), ("n_vocab", C.c_uint32), ("type", C.c_uint32), ("scale", C.c_float)]


class _TokenScores(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("logprob", "entropy", "stat", "top_token", "top_logprob")] + \
               [("n_top", C.c_uint32), ("reserved0", C.c_uint32)]


class _RewardWeights(C.Structure):
    _fields_ = [(n, C.c_float) for n in ("ok", "cons", "real", "safe")]


class _PolicyBatch(C.Structure):
    _fields_ = [("logprob", C.c_void_p), ("logprob_old", C.c_void_p), ("logprob_ref", C.c_void_p), ("n", C.c_uint64),
                ("start", C.c_void_p), ("len", C.c_void_p), ("advantage", C.c_void_p), ("weight", C.c_void_p),
                ("n_sample", C.c_uint32), ("max_len", C.c_uint32), ("log_lo", C.c_float), ("log_hi", C.c_float),
                ("kl", C.c_float), ("reserved0", C.c_uint32)]


_lib = None


def load():
    """Loads the built library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2506_17506_amd.build` (hipcc, gfx950)")
        # torch first: the library must bind to the HIP runtime torch has loaded, so that
        # both see the same device context and allocations
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        L.vl_mir_create.restype = C.c_int32
        L.vl_mir_create.argtypes = [C.c_void_p, C.POINTER(C.c_void_p)]
        L.vl_mir_create_lanes.restype = C.c_int32
        L.vl_mir_create_lanes.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_void_p)]
        L.vl_mir_lanes_get.restype = C.c_int32
        L.vl_mir_lanes_get.argtypes = [C.c_void_p, C.c_void_p]
        L.vl_lanes_expand.restype = C.c_int32
        L.vl_lanes_expand.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32, C.c_uint64, C.c_void_p, C.c_uint64, C.c_void_p]
        L.vl_mir_destroy.restype = None
        L.vl_mir_destroy.argtypes = [C.c_void_p]
        L.vl_liveness_multi.restype = C.c_int32
        L.vl_liveness_multi.argtypes = [C.c_void_p, C.c_uint32, C.c_uint32, C.c_uint32, C.c_void_p, C.c_void_p]
        L.vl_liveness.restype = C.c_int32
        L.vl_liveness.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p, C.POINTER(C.c_void_p)]
        L.vl_live_destroy.restype = None
        L.vl_live_destroy.argtypes = [C.c_void_p]
        L.vl_live_get.restype = C.c_int32
        L.vl_live_get.argtypes = [C.c_void_p, C.c_void_p]
        L.vl_verify_batch.restype = C.c_int32
        L.vl_verify_batch.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint32, C.c_uint64, C.c_void_p, C.c_void_p]
        L.vl_verify_batch_static.restype = C.c_int32
        L.vl_verify_batch_static.argtypes = L.vl_verify_batch.argtypes
        L.vl_verify_multi.restype = C.c_int32
        L.vl_verify_multi.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p]
        L.vl_verify_multi_occ_major.restype = C.c_int32
        L.vl_verify_multi_occ_major.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p]
        L.vl_summarize_multi.restype = C.c_int32
        L.vl_summarize_multi.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.vl_count_violations_multi.restype = C.c_int32
        L.vl_count_violations_multi.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p]
        L.vl_bank_conflicts.restype = C.c_int32
        L.vl_bank_conflicts.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32, C.c_uint64, C.c_uint32, C.c_void_p, C.c_void_p]
        L.vl_free_bases_multi.restype = C.c_int32
        L.vl_free_bases_multi.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p, C.c_void_p]
        L.vl_token_logprobs_work.restype = C.c_int32
        L.vl_token_logprobs_work.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
        L.vl_token_logprobs.restype = C.c_int32
        L.vl_token_logprobs.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
        L.vl_token_logprobs_grad.restype = C.c_int32
        L.vl_token_logprobs_grad.argtypes = [C.c_void_p] * 6 + [C.c_uint64, C.c_void_p]
        L.vl_group_advantages.restype = C.c_int32
        L.vl_group_advantages.argtypes = [C.c_void_p, C.c_void_p, C.c_uint32, C.c_void_p, C.c_uint32, C.c_void_p, C.c_float,
                                          C.c_void_p, C.c_void_p, C.c_void_p]
        L.vl_policy_loss_work.restype = C.c_int32
        L.vl_policy_loss_work.argtypes = [C.c_void_p, C.c_void_p]
        L.vl_policy_loss.restype = C.c_int32
        L.vl_policy_loss.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint64, C.c_void_p]
        L.vl_strerror.restype = C.c_char_p
        L.vl_strerror.argtypes = [C.c_int32]
        L.vl_last_hip_error.restype = C.c_int32
        _lib = L
    return _lib


def vl_strerror(code: int) -> str:
    return load().vl_strerror(code).decode()


def vl_last_hip_error() -> int:
    return int(load().vl_last_hip_error())


def _p(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _stream_ptr(stream):
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return C.c_void_p(int(getattr(stream, "cuda_stream", stream)))


def _u32(what, x, code=-2):
    """a size that a field or an argument of 32 bits holds (of others ctypes would take the low bits)"""
    if x >> 32:
        raise VlError(code, what)
    return x


def make_desc(m):
    """(desc, keepalive) for any object with the array attributes of a program
    description (blk_start, succ_off, succ, instr_occ_off, occ_vreg, occ_flags,
    vreg_class, vreg_width, vreg_align, class_size, class_reserved)."""
    keep = dict(
        blk_start=np.ascontiguousarray(m.blk_start, np.uint32),
        succ_off=np.ascontiguousarray(m.succ_off, np.uint32),
        succ=np.ascontiguousarray(m.succ, np.uint32),
        instr_occ_off=np.ascontiguousarray(m.instr_occ_off, np.uint32),
        occ_vreg=np.ascontiguousarray(m.occ_vreg, np.uint32),
        occ_flags=np.ascontiguousarray(m.occ_flags, np.uint8),
        vreg_class=np.ascontiguousarray(m.vreg_class, np.uint8),
        vreg_width=np.ascontiguousarray(m.vreg_width, np.uint8),
        vreg_align=np.ascontiguousarray(m.vreg_align, np.uint8),
        class_size=np.ascontiguousarray(m.class_size, np.uint16),
        class_reserved=None if getattr(m, "class_reserved", None) is None else
        np.ascontiguousarray(m.class_reserved, np.uint32),
    )
    d = _Desc(len(keep["instr_occ_off"]) - 1, len(keep["vreg_class"]), len(keep["blk_start"]) - 1,
              len(keep["occ_vreg"]), len(keep["class_size"]), len(keep["succ"]),
              *[_p(keep[k]) for k in ("blk_start", "succ_off", "succ", "instr_occ_off", "occ_vreg",
                                      "occ_flags", "vreg_class", "vreg_width", "vreg_align",
                                      "class_size", "class_reserved")])
    return d, keep


def vl_mir_create(m) -> C.c_void_p:
    d, keep = m if isinstance(m, tuple) else make_desc(m)
    out = C.c_void_p()
    rc = load().vl_mir_create(C.byref(d), C.byref(out))
    if rc != 0:
        raise VlError(rc, "vl_mir_create")
    return out


def vl_mir_create_lanes(m, occ_lanes=None) -> C.c_void_p:
    """occ_lanes: uint32 [n_occ] (bit j = lane j, 0 = all) or None; defaults to m.occ_lanes."""
    d, keep = m if isinstance(m, tuple) else make_desc(m)
    if occ_lanes is None and not isinstance(m, tuple):
        occ_lanes = getattr(m, "occ_lanes", None)
    lanes = None if occ_lanes is None else np.ascontiguousarray(occ_lanes, np.uint32)
    out = C.c_void_p()
    rc = load().vl_mir_create_lanes(C.byref(d), _p(lanes), C.byref(out))
    if rc != 0:
        raise VlError(rc, "vl_mir_create_lanes")
    return out


def vl_mir_lanes_get(mir) -> dict:
    """The maps of a handle made by vl_mir_create_lanes, copied to numpy (synchronises)."""
    v = _LanesView()
    rc = load().vl_mir_lanes_get(mir, C.byref(v))
    if rc != 0:
        raise VlError(rc, "vl_mir_lanes_get")
    import torch
    torch.cuda.synchronize()
    hip = hip_runtime()

    def grab(ptr, n, dtype):
        a = np.zeros(n, dtype)
        if ptr and a.nbytes:
            assert hip.hipMemcpy(_p(a), C.c_void_p(ptr), a.nbytes, 2) == 0
        return a
    return dict(n_occ=v.n_occ, n_vreg=v.n_vreg, n_occ_low=v.n_occ_low, n_vreg_low=v.n_vreg_low,
                occ_src=grab(v.occ_src, v.n_occ_low, np.uint32), occ_add=grab(v.occ_add, v.n_occ_low, np.uint8),
                val_vreg=grab(v.val_vreg, v.n_vreg_low, np.uint32), val_lane=grab(v.val_lane, v.n_vreg_low, np.uint8))


def vl_lanes_expand(mir, cand, K: int, ld: int, cand_low, ld_low: int, stream=None) -> None:
    """cand, cand_low: device pointers or tensors of uint16 rows."""
    rc = load().vl_lanes_expand(mir, C.c_void_p(_dev_ptr(cand)), _u32("vl_lanes_expand", K), ld, C.c_void_p(_dev_ptr(cand_low)), ld_low,
                                _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_lanes_expand")


def vl_mir_destroy(mir) -> None:
    load().vl_mir_destroy(mir)


def vl_liveness_multi(mirs, flags: int = 0, tile_len: int = 0, stream=None, live=None):
    """Returns the list of live handles; pass the previous list as `live` to
    reuse its device storage."""
    n = len(mirs)
    arr_m = (C.c_void_p * n)(*[m.value for m in mirs])
    arr_l = (C.c_void_p * n)(*([None] * n if live is None else [l.value for l in live]))
    rc = load().vl_liveness_multi(arr_m, n, flags, tile_len, _stream_ptr(stream), arr_l)
    if rc != 0:
        raise VlError(rc, "vl_liveness_multi")
    return [C.c_void_p(arr_l[k]) for k in range(n)]


def vl_liveness(mir, flags: int = 0, stream=None) -> C.c_void_p:
    out = C.c_void_p()
    rc = load().vl_liveness(mir, flags, _stream_ptr(stream), C.byref(out))
    if rc != 0:
        raise VlError(rc, "vl_liveness")
    return out


def vl_live_destroy(live) -> None:
    load().vl_live_destroy(live)


def vl_live_get(live) -> _View:
    v = _View()
    rc = load().vl_live_get(live, C.byref(v))
    if rc != 0:
        raise VlError(rc, "vl_live_get")
    return v


def vl_verify_batch(mir, live, cand, K: int, ld: int, out, stream=None) -> None:
    """cand, out: device pointers (int) or torch tensors."""
    rc = load().vl_verify_batch(mir, live, C.c_void_p(_dev_ptr(cand)), _u32("vl_verify_batch", K), ld, C.c_void_p(_dev_ptr(out)),
                                _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_verify_batch")


def vl_verify_batch_static(mir, live, cand, K: int, ld: int, out, stream=None) -> None:
    """vl_verify_batch without any allocation inside the library."""
    rc = load().vl_verify_batch_static(mir, live, C.c_void_p(_dev_ptr(cand)), _u32("vl_verify_batch_static", K), ld, C.c_void_p(_dev_ptr(out)),
                                       _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_verify_batch_static")


def make_jobs(jobs):
    """jobs: sequence of (mir, live, cand, K, ld, out) -> ctypes array (reusable)."""
    arr = (_Job * len(jobs))()
    for i, (mir, live, cand, K, ld, out) in enumerate(jobs):
        arr[i].mir, arr[i].live = mir.value, live.value
        arr[i].cand, arr[i].K, arr[i].ld, arr[i].out = _dev_ptr(cand), _u32("make_jobs", K), ld, _dev_ptr(out)
    return arr


def vl_verify_multi(jobs, stream=None) -> None:
    arr = jobs if isinstance(jobs, C.Array) else make_jobs(jobs)
    rc = load().vl_verify_multi(arr, len(arr), _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_verify_multi")


def vl_verify_multi_occ_major(jobs, stream=None) -> None:
    """jobs as for vl_verify_multi, but cand is [n_occ][ld] (occurrence-major), ld >= K."""
    arr = jobs if isinstance(jobs, C.Array) else make_jobs(jobs)
    rc = load().vl_verify_multi_occ_major(arr, len(arr), _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_verify_multi_occ_major")


def vl_summarize_multi(jobs, summaries, stats=None, stream=None) -> None:
    """summaries: device buffer of len(jobs) vl_summary records (24 bytes each); stats:
    device buffer of one vl_loop_stats record (48 bytes) or None."""
    arr = jobs if isinstance(jobs, C.Array) else make_jobs(jobs)
    rc = load().vl_summarize_multi(arr, len(arr), C.c_void_p(_dev_ptr(summaries)),
                                   C.c_void_p(_dev_ptr(stats)) if stats is not None else None, _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_summarize_multi")


COUNTS_DTYPE = np.dtype([("kinds", "<u4"), ("n_cons", "<u4"), ("n_real", "<u4"), ("n_safe", "<u4"), ("real_bits", "<u4"),
                         ("reserved", "<u4", (3,))])


def vl_count_violations_multi(jobs, stream=None) -> None:
    """jobs: sequence of (mir, live, cand, K, ld, out) with out a device buffer of K records
    of 32 bytes (COUNTS_DTYPE)."""
    arr = (_CountJob * len(jobs))()
    for i, (mir, live, cand, K, ld, out) in enumerate(jobs):
        arr[i].mir, arr[i].live = mir.value, live.value
        arr[i].cand, arr[i].K, arr[i].ld, arr[i].out = _dev_ptr(cand), _u32("vl_count_violations_multi", K), ld, _dev_ptr(out)
    rc = load().vl_count_violations_multi(arr, len(arr), _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_count_violations_multi")


def vl_bank_conflicts(mir, cand, K: int, ld: int, n_banks: int, out, stream=None) -> None:
    """out: device buffer of K uint32."""
    rc = load().vl_bank_conflicts(mir, C.c_void_p(_dev_ptr(cand)), _u32("vl_bank_conflicts", K), ld, _u32("vl_bank_conflicts", n_banks, -3), C.c_void_p(_dev_ptr(out)),
                                  _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_bank_conflicts")


def make_mask_queries(queries):
    """queries: sequence of (mir, live, row, occ), row a device pointer or tensor holding one
    candidate row -> ctypes array (reusable)."""
    arr = (_MaskQuery * len(queries))()
    for j, (mir, live, row, occ) in enumerate(queries):
        arr[j].mir, arr[j].live, arr[j].cand, arr[j].occ, arr[j].reserved0 = mir.value, live.value, _dev_ptr(row), occ, 0
    return arr


def vl_free_bases_multi(queries, masks, stream=None) -> None:
    """masks: device buffer of 16 uint32 per query."""
    arr = queries if isinstance(queries, C.Array) else make_mask_queries(queries)
    rc = load().vl_free_bases_multi(arr, len(arr), C.c_void_p(_dev_ptr(masks)), _stream_ptr(stream))
    if rc != 0:
        raise VlError(rc, "vl_free_bases_multi")


# ---- token scores and the policy loss: torch tensors on the current device, from which the sizes are taken

VL_F32, VL_F16, VL_BF16 = 0, 1, 2
VL_MAX_VOCAB, VL_MAX_TOP = 1 << 24, 32
POLICY_STATS_DTYPE = np.dtype([("loss", "<f4"), ("kl", "<f4"), ("n_token", "<u8"), ("n_clipped", "<u8")])   # vl_policy_stats
# the structures' fields as bytes, which is quicker than a ctypes structure per call
_ROWS, _SCORES = struct.Struct("<QQQQQIIIf").pack, struct.Struct("<QQQQQII").pack
_WEIGHTS, _BATCH = struct.Struct("<ffff").pack, struct.Struct("<QQQQQQQQIIfffI").pack
_ELSEWHERE = " (a tensor is not on the current device)"


def _packed(what, pack, *fields):
    try:
        return pack(*fields)
    except (struct.error, OverflowError):   # a size or a number that its field does not hold
        raise VlError(-3, what) from None



class _Torch:
    """what of torch the calls below need, looked up once"""
    def __init__(self):
        import torch
        self.empty, self.uint8 = torch.empty, torch.uint8
        self.type = {torch.float32: VL_F32, torch.float16: VL_F16, torch.bfloat16: VL_BF16}
        self.f32 = (torch.float32,)
        self.words = (torch.int32, torch.uint32)
        self.longs = (torch.int64, torch.uint64)
        self.record = (torch.uint8, torch.int32, torch.uint32, torch.int64)
        self.device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        self.stream = raw or (lambda device: torch.cuda.current_stream(device).cuda_stream)
        self.on, self.external = torch.cuda.stream, torch.cuda.ExternalStream


_t = None


def _device_of(x, what):
    """the current device, which `x` has to be on (tensors of the host and of other devices are refused)"""
    global _t
    if x is None:
        raise VlError(-1, what)
    if _t is None:
        load()
        _t = _Torch()
    device = x.get_device()   # (-1: the host)
    if x.is_cuda and device == _t.device():
        return device
    raise VlError(-7, what + _ELSEWHERE)


def _tensor(what, x, dtypes, shape, device, nullable=True):
    """The pointer of a contiguous tensor of one of the types and that shape (None: of any) on that device, 0 for None."""
    if x is None:
        if nullable:
            return 0
        raise VlError(-1, what)
    if x.get_device() == device and x.dtype in dtypes and (shape is None or x.shape == shape) and x.is_contiguous():
        return x.data_ptr()
    if x.get_device() != device:
        raise VlError(-7, what + _ELSEWHERE)
    raise VlError(-2 if x.dtype in dtypes else -3, what)


def _row_pitch(what, x):
    """distance of the rows of a matrix whose rows are contiguous"""
    if x.dim() == 2:
        ld, step = x.stride()
        if step == 1 or x.shape[1] <= 1:
            return ld
    raise VlError(-2, what)


def _token_rows(what, logits, token, mask, scale):
    """(vl_token_rows as bytes, n_row, n_vocab, device)"""
    device = _device_of(logits, what)
    kind = _t.type.get(logits.dtype)
    if kind is None:
        raise VlError(-3, what)
    ld = _row_pitch(what, logits)
    n, v = logits.shape
    if not n or not v:   # (an empty tensor has no pointer)
        raise VlError(-3 if n else -2, what)
    p_mask = mask_ld = 0
    if mask is not None:
        if mask.get_device() != device:
            raise VlError(-7, what + _ELSEWHERE)
        if mask.dtype not in _t.words:
            raise VlError(-3, what)
        shared = mask.dim() == 1
        if not (shared or (mask.dim() == 2 and mask.shape[0] == n)) or mask.shape[-1] * 32 < v or (mask.stride(-1) != 1 and mask.shape[-1] > 1):
            raise VlError(-2, what)
        p_mask, mask_ld = mask.data_ptr(), 0 if shared or n == 1 else mask.stride(0)
    p_token = 0 if token is None else _tensor(what, token, _t.words[:1], (n,), device)
    return _packed(what, _ROWS, logits.data_ptr(), ld, p_mask, mask_ld, p_token, n, v, kind, scale), n, v, device


def _call_stream(stream, device):
    return _t.stream(device) if stream is None else int(getattr(stream, "cuda_stream", getattr(stream, "value", stream)) or 0)


def _bytes_of(what, call, *args):
    need = C.c_uint64()
    rc = call(*args, C.byref(need))
    if rc != 0:
        raise VlError(rc, what)
    return need.value


def _work(what, n_bytes, work, stream, device):
    """(pointer, bytes, the tensor): `work`, or n_bytes of the call's own, allocated on the stream it runs on"""
    if work is not None:
        if work.get_device() != device:
            raise VlError(-7, what + _ELSEWHERE)
        if not work.is_contiguous():
            raise VlError(-2, what)
    elif not n_bytes:
        return None, 0, None
    elif stream is None:
        work = _t.empty(n_bytes, dtype=_t.uint8, device=device)
    else:
        with _t.on(stream if hasattr(stream, "cuda_stream") else _t.external(_call_stream(stream, device), device=device)):
            work = _t.empty(n_bytes, dtype=_t.uint8, device=device)
    return work.data_ptr(), work.numel() * work.element_size(), work


def _token_scores(logits, token, mask, scale, logprob, entropy, stat, top_token, top_logprob):
    """(vl_token_rows, vl_token_scores as bytes, device)"""
    what = "vl_token_logprobs"
    rows, n, _, device = _token_rows(what, logits, token, mask, scale)
    f, k = _t.f32, 0
    some = top_token if top_token is not None else top_logprob
    if some is not None:
        if some.dim() != 2:
            raise VlError(-2, what)
        k = some.shape[1]
    return rows, _packed(what, _SCORES, _tensor(what, logprob, f, (n,), device), _tensor(what, entropy, f, (n,), device), _tensor(what, stat, f, (n, 2), device),
                              _tensor(what, top_token, _t.words[:1], (n, k), device), _tensor(what, top_logprob, f, (n, k), device), k, 0), device


def vl_token_logprobs_work(logits, token=None, mask=None, scale=1.0, logprob=None, entropy=None, stat=None, top_token=None,
                           top_logprob=None) -> int:
    """Bytes of work that vl_token_logprobs needs for the same arguments."""
    rows, out, _ = _token_scores(logits, token, mask, scale, logprob, entropy, stat, top_token, top_logprob)
    return _bytes_of("vl_token_logprobs_work", load().vl_token_logprobs_work, rows, out)


def vl_token_logprobs(logits, token=None, mask=None, scale=1.0, logprob=None, entropy=None, stat=None, top_token=None,
                      top_logprob=None, work=None, stream=None) -> None:
    """logits [n_row, n_vocab] in float32, float16 or bfloat16, rows of any pitch (a window of the columns of wider rows is
    one); token int32 [n_row]; mask int32 words [n_row, words] or [words] for all rows.  Written, those that are given:
    logprob, entropy float32 [n_row], stat float32 [n_row, 2], top_token int32 and top_logprob float32 [n_row, n_top].
    work: memory of vl_token_logprobs_work bytes, allocated on the call's stream if not given."""
    what = "vl_token_logprobs"
    rows, out, device = _token_scores(logits, token, mask, scale, logprob, entropy, stat, top_token, top_logprob)
    p, n_bytes, keep = _work(what, 0 if work is not None else _bytes_of(what, _lib.vl_token_logprobs_work, rows, out), work, stream, device)
    rc = _lib.vl_token_logprobs(rows, out, p, n_bytes, _call_stream(stream, device))
    if rc != 0:
        raise VlError(rc, what)


def vl_token_logprobs_grad(logits, stat, grad, token=None, mask=None, scale=1.0, entropy=None, g_logprob=None, g_entropy=None,
                           stream=None) -> None:
    """grad [n_row, n_vocab] of the logits' type and any pitch, or logits itself; stat and entropy as vl_token_logprobs wrote
    them for the same rows; g_logprob, g_entropy float32 [n_row]."""
    what = "vl_token_logprobs_grad"
    rows, n, _, device = _token_rows(what, logits, token, mask, scale)
    if grad is None:
        raise VlError(-1, what)
    if grad.get_device() != device:
        raise VlError(-7, what + _ELSEWHERE)
    if grad.dtype != logits.dtype:
        raise VlError(-3, what)
    if grad.shape != logits.shape:
        raise VlError(-2, what)
    f = _t.f32
    rc = _lib.vl_token_logprobs_grad(rows, _tensor(what, stat, f, (n, 2), device), _tensor(what, entropy, f, (n,), device),
                                     _tensor(what, g_logprob, f, (n,), device), _tensor(what, g_entropy, f, (n,), device),
                                     grad.data_ptr(), _row_pitch(what, grad), _call_stream(stream, device))
    if rc != 0:
        raise VlError(rc, what)


def vl_group_advantages(counts, group_off, weights, eps, advantage, reward=None, extra=None, stream=None) -> None:
    """counts: the records vl_count_violations_multi wrote (int32 [n, 8] or 32 n bytes) or None; group_off int32 [n_group + 1];
    weights: (ok, cons, real, safe); advantage, reward, extra float32 [n]."""
    what = "vl_group_advantages"
    device = _device_of(group_off, what)
    some = advantage if advantage is not None else reward if reward is not None else extra
    if some is None:
        raise VlError(-1, what)
    shape, n, n_group, f = some.shape, some.numel(), max(0, group_off.numel() - 1), _t.f32
    if not n or n >> 31 or n_group >> 31:   # (the arguments of 32 bits would take the low ones)
        raise VlError(-2, what)
    p = _tensor(what, counts, _t.record[:3], None, device)
    if counts is not None and counts.numel() * counts.element_size() != 32 * n:
        raise VlError(-2, what)
    rc = _lib.vl_group_advantages(p, _tensor(what, extra, f, shape, device), n, _tensor(what, group_off, _t.words, None, device),
                                  n_group, _packed(what, _WEIGHTS, *weights), eps, _tensor(what, reward, f, shape, device),
                                  _tensor(what, advantage, f, shape, device), _call_stream(stream, device))
    if rc != 0:
        raise VlError(rc, what)


def _policy_batch(logprob, logprob_old, start, length, advantage, weight, log_lo, log_hi, logprob_ref, kl, max_len):
    """(vl_policy_batch as bytes, device)"""
    what = "vl_policy_loss"
    device = _device_of(logprob, what)
    if start is None:
        raise VlError(-1, what)
    f, shape, samples, n = _t.f32, logprob.shape, start.shape, logprob.numel()
    m = start.numel()
    if not n or not m:
        raise VlError(-2, what)
    if max_len is None:   # the mean length, if there is no room between the samples: a launch's shape, not a bound
        max_len = min(0xFFFFFFFF, n // max(1, m) + 1)
    return _packed(what, _BATCH, _tensor(what, logprob, f, None, device), _tensor(what, logprob_old, f, shape, device, False),
                       _tensor(what, logprob_ref, f, shape, device), n, _tensor(what, start, _t.longs, None, device),
                       _tensor(what, length, _t.words, samples, device, False), _tensor(what, advantage, f, samples, device, False),
                       _tensor(what, weight, f, samples, device, False), m, max_len, log_lo, log_hi, kl, 0), device


def vl_policy_loss_work(logprob, logprob_old, start, length, advantage, weight, log_lo, log_hi, logprob_ref=None, kl=0.0,
                        max_len=None) -> int:
    """Bytes of work that vl_policy_loss needs for the same arguments."""
    batch, _ = _policy_batch(logprob, logprob_old, start, length, advantage, weight, log_lo, log_hi, logprob_ref, kl, max_len)
    return _bytes_of("vl_policy_loss_work", load().vl_policy_loss_work, batch)


def vl_policy_loss(logprob, logprob_old, start, length, advantage, weight, grad, stats, log_lo, log_hi, logprob_ref=None, kl=0.0,
                   max_len=None, work=None, stream=None) -> None:
    """logprob, logprob_old, logprob_ref, grad: float32 of one shape; start int64, length int32, advantage, weight float32
    [n_sample]; stats: device buffer of one POLICY_STATS_DTYPE record (24 bytes); max_len: the longest sample if known."""
    what = "vl_policy_loss"
    batch, device = _policy_batch(logprob, logprob_old, start, length, advantage, weight, log_lo, log_hi, logprob_ref, kl, max_len)
    p_grad = _tensor(what, grad, _t.f32, logprob.shape, device, False)
    p_stats = _tensor(what, stats, _t.record, None, device, False)
    if stats.numel() * stats.element_size() < 24:
        raise VlError(-2, what)
    p, n_bytes, keep = _work(what, 0 if work is not None else _bytes_of(what, _lib.vl_policy_loss_work, batch), work, stream, device)
    rc = _lib.vl_policy_loss(batch, p_grad, p_stats, p, n_bytes, _call_stream(stream, device))
    if rc != 0:
        raise VlError(rc, what)


def _dev_ptr(x) -> int:
    return int(x.data_ptr()) if hasattr(x, "data_ptr") else int(x)


# ---- helpers around torch device memory (no arithmetic of the method) ----

def pad_ld(n_occ: int) -> int:
    """Row pitch in elements: rows start on 128-byte lines."""
    return max(64, (n_occ + 63) // 64 * 64)


def rows_to_device(rows: np.ndarray, device="cuda"):
    """uint16 [K, O] host rows -> (int16 device tensor [K, ld], ld)."""
    import torch
    K, O = rows.shape
    ld = pad_ld(O)
    host = np.zeros((K, ld), np.uint16)
    host[:, :O] = rows
    return torch.from_numpy(host.view(np.int16)).to(device), ld


_hip = None


def hip_runtime():
    """The HIP runtime library already mapped into this process (torch's)."""
    global _hip
    if _hip is None:
        import torch  # noqa: F401
        path = "libamdhip64.so"
        with open("/proc/self/maps") as f:
            for line in f:
                if "libamdhip64" in line:
                    path = line.split()[-1]
                    break
        _hip = C.CDLL(path)
        _hip.hipMemcpy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int]
        _hip.hipEventCreate.argtypes = [C.POINTER(C.c_void_p)]
        _hip.hipEventDestroy.argtypes = [C.c_void_p]
        _hip.hipEventElapsedTime.argtypes = [C.POINTER(C.c_float), C.c_void_p, C.c_void_p]
    return _hip


def view_to_numpy(v: _View) -> dict:
    """Copies the device arrays of a live view to numpy (synchronises)."""
    import torch
    torch.cuda.synchronize()
    hip = hip_runtime()

    def grab(ptr, shape, dtype):
        a = np.zeros(shape, dtype)
        if ptr and a.nbytes:
            rc = hip.hipMemcpy(_p(a), C.c_void_p(ptr), a.nbytes, 2)
            if rc != 0:
                raise RuntimeError(f"hipMemcpy failed: {rc}")
        return a
    W = v.words
    out = dict(
        live_in=grab(v.live_in, (v.n_block, W), np.uint32),
        live_out=grab(v.live_out, (v.n_block, W), np.uint32),
        occ_kill=grab(v.occ_kill, (v.n_occ,), np.uint8),
        seg_off=grab(v.seg_off, (v.n_vreg + 1,), np.uint32),
        seg=grab(v.seg, (v.n_seg, 2), np.uint32),
        hull=grab(v.hull, (v.n_vreg, 2), np.uint32),
    )
    out["live_after"] = grab(v.live_after, (v.n_instr, W), np.uint32) if v.live_after else None
    return out
