"""ctypes binding of ``include/nms.h``: argument marshalling only.

Tensor arguments are torch tensors on the GPU (device memory is torch's job);
their ``data_ptr()`` and the current torch HIP stream are handed to the C ABI.
Every function returns nothing and raises :class:`NmsError` on a non-zero status.
"""
from __future__ import annotations

import ctypes
import os

# torch first: its wheel carries its own HIP runtime (soname libamdhip64.so.7).  Once
# that copy is in the process the loader binds the library below to it; loaded the other
# way round, the system runtime would come in as a second, unusable instance.
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libnms_mi355x.so")

NMS_OK = 0
NMS_ERR_INVALID_ARG = -1
NMS_ERR_TOO_LARGE = -2
NMS_ERR_WORKSPACE = -3
NMS_ERR_LAUNCH = -4
NMS_ROUTE_DIRECT, NMS_ROUTE_ALL_PAIRS, NMS_ROUTE_TWO_LAUNCH, NMS_ROUTE_EARLY_EXIT, NMS_ROUTE_SMALL_FRAMES = 0, 1, 2, 3, 4
NMS_ROUTE_PLACE_FRAMES, NMS_ROUTE_PLACE_TABLE = 5, 6

EXPORTS = (
    "nms_status_string", "nms_version", "nms_last_launch_error", "nms_padded_n", "nms_mask_words",
    "nms_sort_workspace_bytes", "nms_workspace_bytes", "nms_route", "nms_route_at",
    "nms_sort", "nms_sort_batched", "nms_overlap_mask", "nms_overlap_mask_batched",
    "nms_reduce", "nms_reduce_batched", "nms_run_ws", "nms_run_batched", "nms_run_ranked_batched", "nms_run_direct_batched",
    "nms_run_batched_profiled", "nms_reduce_greedy", "nms_reduce_greedy_batched",
    "nms_greedy_workspace_bytes", "nms_run_greedy_batched", "nms_run_greedy_fused_batched", "nms_run_early_exit_batched", "nms_map_matrix", "nms_reduce_matrix",
    "nms_ex_workspace_bytes", "nms_run_ex_batched",
    "nms_init", "nms_shutdown", "nms_run", "nms_run_static_batched", "nms_host_pair_test",
    "nms_verify_workspace_bytes", "nms_verify_batched", "nms_cache_moves_max", "nms_cache_workspace_bytes",
    "nms_cache_keep_batched", "nms_cache_move_batched", "nms_cache_evict_batched",
)


class NmsOptions(ctypes.Structure):
    """struct nms_options of include/nms.h."""
    _fields_ = [("rule", ctypes.c_int32), ("measure", ctypes.c_int32), ("compare", ctypes.c_int32),
                ("ties", ctypes.c_int32), ("pixel_offset", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("classes", ctypes.c_void_p)]


class NmsCacheWeights(ctypes.Structure):
    """struct nms_cache_weights of include/nms.h."""
    _fields_ = [("weights", ctypes.c_void_p), ("row_stride", ctypes.c_longlong), ("type", ctypes.c_int32),
                ("group", ctypes.c_int32), ("tokens", ctypes.c_int32), ("columns", ctypes.c_int32),
                ("valid_tokens", ctypes.c_void_p)]


class NmsCacheTensor(ctypes.Structure):
    """struct nms_cache_tensor of include/nms.h."""
    _fields_ = [("rows", ctypes.c_void_p), ("row_bytes", ctypes.c_longlong), ("sequence_stride", ctypes.c_longlong),
                ("head_stride", ctypes.c_longlong), ("slot_stride", ctypes.c_longlong)]


class NmsCachePages(ctypes.Structure):
    """struct nms_cache_pages of include/nms.h."""
    _fields_ = [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int32), ("page_slots", ctypes.c_int32),
                ("pages", ctypes.c_int32), ("reserved", ctypes.c_int32)]


RULES = {"paper": 0, "greedy": 1}
MEASURES = {"outranking_area": 0, "iou": 1}
COMPARES = {"ge": 0, "gt": 1}
TIES = {"index": 0, "ignore": 1}


class NmsError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        detail = f" [{lib.nms_last_launch_error().decode()}]" if status == NMS_ERR_LAUNCH else ""
        super().__init__(f"{where}: {nms_status_string(status)} ({status}){detail}")


def library_path() -> str:
    return _LIB_PATH


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2502_00535_amd.build` "
            "(there is no CPU fallback)")
    L = ctypes.CDLL(_LIB_PATH)
    vp, i32, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    L.nms_status_string.restype = ctypes.c_char_p
    L.nms_status_string.argtypes = [i32]
    L.nms_version.restype = i32
    L.nms_version.argtypes = []
    L.nms_last_launch_error.restype = ctypes.c_char_p
    L.nms_last_launch_error.argtypes = []
    L.nms_padded_n.restype = i32
    L.nms_padded_n.argtypes = [i32]
    L.nms_mask_words.restype = sz
    L.nms_mask_words.argtypes = [i32]
    L.nms_sort_workspace_bytes.restype = sz
    L.nms_sort_workspace_bytes.argtypes = [i32, i32]
    L.nms_workspace_bytes.restype = sz
    L.nms_workspace_bytes.argtypes = [i32, i32]
    L.nms_route.restype = i32
    L.nms_route.argtypes = [i32, i32]
    L.nms_route_at.restype = i32
    L.nms_route_at.argtypes = [i32, i32, f32]
    L.nms_sort.restype = i32
    L.nms_sort.argtypes = [vp, vp, i32, vp, vp, vp, sz, vp]
    L.nms_sort_batched.restype = i32
    L.nms_sort_batched.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, sz, vp]
    L.nms_overlap_mask.restype = i32
    L.nms_overlap_mask.argtypes = [vp, i32, f32, vp, vp]
    L.nms_overlap_mask_batched.restype = i32
    L.nms_overlap_mask_batched.argtypes = [vp, vp, i32, i32, f32, vp, vp]
    L.nms_reduce.restype = i32
    L.nms_reduce.argtypes = [vp, vp, i32, vp, vp]
    L.nms_reduce_batched.restype = i32
    L.nms_reduce_batched.argtypes = [vp, vp, vp, i32, i32, vp, vp]
    L.nms_run_ws.restype = i32
    L.nms_run_ws.argtypes = [vp, vp, i32, f32, vp, vp, sz, vp]
    L.nms_run_batched.restype = i32
    L.nms_run_batched.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp, sz, vp]
    L.nms_run_ranked_batched.restype = i32
    L.nms_run_ranked_batched.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp, sz, vp]
    L.nms_run_direct_batched.restype = i32
    L.nms_run_direct_batched.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp]
    L.nms_reduce_greedy.restype = i32
    L.nms_reduce_greedy.argtypes = [vp, vp, i32, vp, vp]
    L.nms_reduce_greedy_batched.restype = i32
    L.nms_reduce_greedy_batched.argtypes = [vp, vp, vp, i32, i32, vp, vp]
    L.nms_greedy_workspace_bytes.restype = sz
    L.nms_greedy_workspace_bytes.argtypes = [i32, i32]
    L.nms_run_greedy_batched.restype = i32
    L.nms_run_greedy_batched.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp, sz, vp]
    L.nms_run_greedy_fused_batched.restype = i32
    L.nms_run_greedy_fused_batched.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp, sz, vp]
    L.nms_run_early_exit_batched.restype = i32
    L.nms_run_early_exit_batched.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp, sz, vp]
    L.nms_run_batched_profiled.restype = i32
    L.nms_run_batched_profiled.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp, sz, vp, ctypes.POINTER(vp)]
    L.nms_map_matrix.restype = i32
    L.nms_map_matrix.argtypes = [vp, vp, i32, i32, f32, vp, vp]
    L.nms_reduce_matrix.restype = i32
    L.nms_reduce_matrix.argtypes = [vp, i32, i32, vp, vp]
    L.nms_ex_workspace_bytes.restype = sz
    L.nms_ex_workspace_bytes.argtypes = [i32, i32]
    L.nms_run_ex_batched.restype = i32
    L.nms_run_ex_batched.argtypes = [vp, vp, vp, i32, i32, f32, ctypes.POINTER(NmsOptions), vp, vp, sz, vp]
    L.nms_init.restype = i32
    L.nms_init.argtypes = [i32, i32, vp, sz]
    L.nms_shutdown.restype = i32
    L.nms_shutdown.argtypes = []
    L.nms_run.restype = i32
    L.nms_run.argtypes = [vp, vp, i32, f32, vp, vp]
    L.nms_run_static_batched.restype = i32
    L.nms_run_static_batched.argtypes = [vp, vp, vp, i32, i32, f32, vp, vp]
    i64 = ctypes.c_longlong
    L.nms_verify_workspace_bytes.restype = sz
    L.nms_verify_workspace_bytes.argtypes = [i32, i32]
    L.nms_verify_batched.restype = i32
    L.nms_verify_batched.argtypes = [vp, i64, vp, i64, i32, vp, vp, i32, i32, i32, vp, vp, vp, vp, sz, vp]
    L.nms_cache_moves_max.restype = i32
    L.nms_cache_moves_max.argtypes = [i32, i32]
    L.nms_cache_workspace_bytes.restype = sz
    L.nms_cache_workspace_bytes.argtypes = [i32, i32, i32, i32]
    weights_p, tensor_p, pages_p = (ctypes.POINTER(s) for s in (NmsCacheWeights, NmsCacheTensor, NmsCachePages))
    L.nms_cache_keep_batched.restype = i32
    L.nms_cache_keep_batched.argtypes = [vp, vp, vp, vp, i32, i32, i32, weights_p, i32, i32, i32, vp, vp, vp, vp, sz, vp]
    L.nms_cache_move_batched.restype = i32
    L.nms_cache_move_batched.argtypes = [vp, i32, i32, i32, i32, tensor_p, i32, pages_p, vp]
    L.nms_cache_evict_batched.restype = i32
    L.nms_cache_evict_batched.argtypes = [vp, vp, vp, vp, i32, i32, i32, weights_p, i32, i32, i32, tensor_p, i32, pages_p,
                                          vp, vp, vp, sz, vp]
    L.nms_host_pair_test.restype = i32
    L.nms_host_pair_test.argtypes = [ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float), f32]
    return L


lib = _load()


# ------------------------------------------------------------------ marshalling helpers

def _on_device(t) -> bool:
    return t.is_cuda


# A call on a small frame is as long as its marshalling (10 us of it at 360 boxes before the helpers below
# compared dtypes as objects, passed addresses as plain integers and asked for the raw stream): they
# build nothing that the call does not need, and look at what is in order in one expression.  The whole-path calls on
# one frame and on batches go through _marshal (csrc/marshal.c), which does the same in native code.
_Tensor = torch.Tensor
_DTYPES = {"float32": torch.float32, "int32": torch.int32, "int64": torch.int64, "uint8": torch.uint8}


def _ptr(t, dtype_name: str | None, what: str, need: int = 0):
    """Device pointer of a contiguous CUDA/HIP tensor (None -> NULL).  `need` is the number
    of elements the library will read or write there: the C ABI takes bare pointers and
    cannot know a buffer's size, so a tensor that is too small is refused here, before a
    kernel could run past its end."""
    if t is None:
        return None
    if (isinstance(t, _Tensor) and t.is_cuda and t.is_contiguous() and t.numel() >= need
            and (dtype_name is None or t.dtype == _DTYPES[dtype_name])):
        return t.data_ptr()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch tensor")
    if t.numel() < need:
        raise ValueError(f"{what}: {t.numel()} elements, the call needs {need}")
    if not _on_device(t):
        raise ValueError(f"{what}: tensor must live on the GPU")
    if not t.is_contiguous():
        raise ValueError(f"{what}: tensor must be contiguous")
    if dtype_name is not None and t.dtype != _DTYPES[dtype_name]:
        raise TypeError(f"{what}: expected dtype {dtype_name}, got {t.dtype}")
    return t.data_ptr()


def _boxes(n_max, frames):
    """frames * n_max, the element count of the per-box buffers; 0 when the library will refuse the sizes anyway."""
    if type(n_max) is not int or type(frames) is not int:
        n_max, frames = int(n_max), int(frames)
    return frames * n_max if n_max >= 0 and frames >= 0 else 0


def _sizes(n_max, frames):
    """Element counts of the per-frame buffers for a batch: (frames * n_max, frames * n_pad,
    frames * mask words); zeros when the library will refuse the sizes anyway."""
    n_max, frames = int(n_max), int(frames)
    if n_max < 0 or frames < 0:
        return 0, 0, 0
    return frames * n_max, frames * int(lib.nms_padded_n(n_max)), frames * int(lib.nms_mask_words(n_max))


def _ws(t):
    if t is None:
        return None, 0
    return _ptr(t, None, "workspace"), t.nbytes


# The current stream's handle without a Stream object around it, where this torch has that (it is not part of
# torch's public interface, so another version may lack it).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)  # torch.cuda.current_device without its check for an initialized runtime


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    if _current_device is None or not torch.cuda.is_initialized():
        return _raw_stream(torch.cuda.current_device())
    return _raw_stream(_current_device())


try:
    from . import _marshal  # noqa: E402  (built with the library)
except ImportError:  # another Python than the one it was built for, or no C compiler there: the calls are marshalled below then
    _marshal = None

if _marshal is not None:
    _marshal.setup(torch.Tensor, torch.float32, torch.int32, torch.uint8, _current_device, _raw_stream)
    _native = _marshal.run
else:
    def _native(*args):
        return None


def _address(name):
    return ctypes.cast(getattr(lib, name), ctypes.c_void_p).value


_RUN_BATCHED, _RUN_RANKED, _RUN_GREEDY = (_address(n) for n in ("nms_run_batched", "nms_run_ranked_batched", "nms_run_greedy_batched"))


def _check(status: int, where: str):
    if status != NMS_OK:
        raise NmsError(status, where)


# ------------------------------------------------------------------ host-only helpers

def nms_status_string(status: int) -> str:
    return lib.nms_status_string(int(status)).decode()


def nms_version() -> int:
    return int(lib.nms_version())


def nms_padded_n(n: int) -> int:
    return int(lib.nms_padded_n(int(n)))


def nms_mask_words(n: int) -> int:
    return int(lib.nms_mask_words(int(n)))


def nms_sort_workspace_bytes(n_max: int, frames: int) -> int:
    return int(lib.nms_sort_workspace_bytes(int(n_max), int(frames)))


def nms_workspace_bytes(n_max: int, frames: int) -> int:
    return int(lib.nms_workspace_bytes(int(n_max), int(frames)))


def nms_route(n_max: int, frames: int) -> int:
    return int(lib.nms_route(int(n_max), int(frames)))


def nms_route_at(n_max: int, frames: int, threshold: float) -> int:
    return int(lib.nms_route_at(int(n_max), int(frames), float(threshold)))


def nms_host_pair_test(victim, outranking, threshold: float) -> int:
    v = (ctypes.c_float * 4)(*[float(x) for x in victim])
    c = (ctypes.c_float * 4)(*[float(x) for x in outranking])
    return int(lib.nms_host_pair_test(v, c, float(threshold)))


# ------------------------------------------------------------------ device entry points

def nms_sort(boxes, scores, n, order, sorted5, workspace=None, stream=None):
    fn_, fp_, fm_ = _sizes(n, 1)
    w, wb = _ws(workspace)
    _check(lib.nms_sort(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_), int(n),
                        _ptr(order, "int32", "order", fn_), _ptr(sorted5, "float32", "sorted5", 5 * fp_),
                        w, wb, _stream(stream)), "nms_sort")


def nms_sort_batched(boxes, scores, counts, n_max, frames, order, sorted5, workspace=None, stream=None):
    fn_, fp_, fm_ = _sizes(n_max, frames)
    w, wb = _ws(workspace)
    _check(lib.nms_sort_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames),
                                _ptr(order, "int32", "order", fn_), _ptr(sorted5, "float32", "sorted5", 5 * fp_),
                                w, wb, _stream(stream)), "nms_sort_batched")


def nms_overlap_mask(sorted5, n, threshold, mask, stream=None):
    fn_, fp_, fm_ = _sizes(n, 1)
    _check(lib.nms_overlap_mask(_ptr(sorted5, "float32", "sorted5", 5 * fp_), int(n), float(threshold),
                                _ptr(mask, "int64", "mask", fm_), _stream(stream)), "nms_overlap_mask")


def nms_overlap_mask_batched(sorted5, counts, n_max, frames, threshold, mask, stream=None):
    fn_, fp_, fm_ = _sizes(n_max, frames)
    _check(lib.nms_overlap_mask_batched(_ptr(sorted5, "float32", "sorted5", 5 * fp_), _ptr(counts, "int32", "counts", int(frames)),
                                        int(n_max), int(frames), float(threshold),
                                        _ptr(mask, "int64", "mask", fm_), _stream(stream)), "nms_overlap_mask_batched")


def nms_reduce(mask, order, n, keep_out, stream=None):
    fn_, fp_, fm_ = _sizes(n, 1)
    _check(lib.nms_reduce(_ptr(mask, "int64", "mask", fm_), _ptr(order, "int32", "order", fn_), int(n),
                          _ptr(keep_out, "uint8", "keep_out", fn_), _stream(stream)), "nms_reduce")


def nms_reduce_batched(mask, order, counts, n_max, frames, keep_out, stream=None):
    fn_, fp_, fm_ = _sizes(n_max, frames)
    _check(lib.nms_reduce_batched(_ptr(mask, "int64", "mask", fm_), _ptr(order, "int32", "order", fn_),
                                  _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames),
                                  _ptr(keep_out, "uint8", "keep_out", fn_), _stream(stream)), "nms_reduce_batched")


def nms_run_ws(boxes, scores, n, threshold, keep_out, workspace, stream=None):
    status = _native(_RUN_BATCHED, boxes, scores, None, n, 1, threshold, keep_out, workspace, stream)  # what nms_run_ws calls
    if status == NMS_OK:
        return
    if status is not None:
        raise NmsError(status, "nms_run_ws")
    fn_ = _boxes(n, 1)
    w, wb = _ws(workspace)
    _check(lib.nms_run_ws(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_), int(n),
                          float(threshold), _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream)),
           "nms_run_ws")


def nms_run_batched(boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream=None):
    status = _native(_RUN_BATCHED, boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream)
    if status == NMS_OK:
        return
    if status is not None:
        raise NmsError(status, "nms_run_batched")
    fn_ = _boxes(n_max, frames)
    w, wb = _ws(workspace)
    _check(lib.nms_run_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                               _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                               _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream)), "nms_run_batched")


class RunPlan:
    """nms_run_batched (or another entry point with the same arguments) with its arguments marshalled once.

    For serving loops that call the library many times on the same buffers: the tensors
    are validated and their pointers taken at construction; each call is then a single
    foreign call.  The plan holds references to its tensors, and uses the stream that was
    current when it was built unless one is given.
    """

    SAME_SIGNATURE = ("nms_run_batched", "nms_run_ranked_batched", "nms_run_early_exit_batched",
                      "nms_run_greedy_batched", "nms_run_greedy_fused_batched")

    def __init__(self, boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream=None,
                 entry="nms_run_batched"):
        if entry not in self.SAME_SIGNATURE:
            raise ValueError(f"RunPlan: {entry} does not take nms_run_batched's arguments")
        self._entry = entry
        self._keepalive = (boxes, scores, counts, keep_out, workspace)
        w, wb = _ws(workspace)
        fn_ = _boxes(n_max, frames)
        self._args = (_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                      _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                      _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream))
        self._fn = getattr(lib, entry)

    def __call__(self):
        status = self._fn(*self._args)
        if status != NMS_OK:
            raise NmsError(status, self._entry)


def nms_run_ranked_batched(boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream=None):
    status = _native(_RUN_RANKED, boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream)
    if status == NMS_OK:
        return
    if status is not None:
        raise NmsError(status, "nms_run_ranked_batched")
    fn_ = _boxes(n_max, frames)
    w, wb = _ws(workspace)
    _check(lib.nms_run_ranked_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                      _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                                      _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream)),
           "nms_run_ranked_batched")


def nms_run_direct_batched(boxes, scores, counts, n_max, frames, threshold, keep_out, stream=None):
    fn_ = _boxes(n_max, frames)
    _check(lib.nms_run_direct_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                      _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                                      _ptr(keep_out, "uint8", "keep_out", fn_), _stream(stream)),
           "nms_run_direct_batched")


def nms_run_batched_profiled(boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, events, stream=None):
    fn_ = _boxes(n_max, frames)
    """events: three raw hipEvent_t handles (ints) or None entries."""
    w, wb = _ws(workspace)
    ev = (ctypes.c_void_p * 3)(*[ctypes.c_void_p(e) if e else None for e in events])
    _check(lib.nms_run_batched_profiled(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                        _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                                        _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream), ev),
           "nms_run_batched_profiled")


def nms_reduce_greedy(mask, order, n, keep_out, stream=None):
    fn_, fp_, fm_ = _sizes(n, 1)
    _check(lib.nms_reduce_greedy(_ptr(mask, "int64", "mask", fm_), _ptr(order, "int32", "order", fn_), int(n),
                                 _ptr(keep_out, "uint8", "keep_out", fn_), _stream(stream)), "nms_reduce_greedy")


def nms_reduce_greedy_batched(mask, order, counts, n_max, frames, keep_out, stream=None):
    fn_, fp_, fm_ = _sizes(n_max, frames)
    _check(lib.nms_reduce_greedy_batched(_ptr(mask, "int64", "mask", fm_), _ptr(order, "int32", "order", fn_),
                                         _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames),
                                         _ptr(keep_out, "uint8", "keep_out", fn_), _stream(stream)),
           "nms_reduce_greedy_batched")


def nms_greedy_workspace_bytes(n_max: int, frames: int) -> int:
    return int(lib.nms_greedy_workspace_bytes(int(n_max), int(frames)))


def nms_run_greedy_batched(boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream=None):
    status = _native(_RUN_GREEDY, boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream)
    if status == NMS_OK:
        return
    if status is not None:
        raise NmsError(status, "nms_run_greedy_batched")
    fn_ = _boxes(n_max, frames)
    w, wb = _ws(workspace)
    _check(lib.nms_run_greedy_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                      _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                                      _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream)),
           "nms_run_greedy_batched")


def nms_run_early_exit_batched(boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream=None):
    fn_ = _boxes(n_max, frames)
    w, wb = _ws(workspace)
    _check(lib.nms_run_early_exit_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                          _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                                          _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream)),
           "nms_run_early_exit_batched")


def nms_run_greedy_fused_batched(boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, stream=None):
    fn_ = _boxes(n_max, frames)
    w, wb = _ws(workspace)
    _check(lib.nms_run_greedy_fused_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                            _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                                            _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream)),
           "nms_run_greedy_fused_batched")


def nms_map_matrix(boxes, scores, n, capacity, threshold, B, stream=None):
    cap = max(int(capacity), 0)
    _check(lib.nms_map_matrix(_ptr(boxes, "float32", "boxes", 4 * max(int(n), 0)),
                              _ptr(scores, "float32", "scores", max(int(n), 0)), int(n),
                              int(capacity), float(threshold), _ptr(B, "uint8", "B", cap * cap), _stream(stream)),
           "nms_map_matrix")


def nms_reduce_matrix(B, capacity, k, V, stream=None):
    cap = max(int(capacity), 0)
    _check(lib.nms_reduce_matrix(_ptr(B, "uint8", "B", cap * cap), int(capacity), int(k), _ptr(V, "uint8", "V", cap),
                                 _stream(stream)), "nms_reduce_matrix")


def nms_ex_workspace_bytes(n_max: int, frames: int) -> int:
    return int(lib.nms_ex_workspace_bytes(int(n_max), int(frames)))


def nms_run_ex_batched(boxes, scores, counts, n_max, frames, threshold, keep_out, workspace, rule="paper",
                       measure="outranking_area", compare="ge", ties="index", pixel_offset=1.0, classes=None,
                       stream=None):
    fn_ = _boxes(n_max, frames)
    w, wb = _ws(workspace)
    cls = _ptr(classes, "int32", "classes", fn_)
    opt = NmsOptions(RULES[rule], MEASURES[measure], COMPARES[compare], TIES[ties], float(pixel_offset), 0,
                     cls)
    _check(lib.nms_run_ex_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                  _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                                  ctypes.byref(opt), _ptr(keep_out, "uint8", "keep_out", fn_), w, wb, _stream(stream)),
           "nms_run_ex_batched")


def nms_init(n_max, frames_max, workspace):
    w, wb = _ws(workspace)
    _check(lib.nms_init(int(n_max), int(frames_max), w, wb), "nms_init")


def nms_shutdown():
    _check(lib.nms_shutdown(), "nms_shutdown")


def nms_run(boxes, scores, n, threshold, keep_out, stream=None):
    fn_ = _boxes(n, 1)
    _check(lib.nms_run(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_), int(n),
                       float(threshold), _ptr(keep_out, "uint8", "keep_out", fn_), _stream(stream)), "nms_run")


NMS_STATIC_SCRATCH_BYTES = 4194304


def nms_run_static_batched(boxes, scores, counts, n_max, frames, threshold, keep_out, stream=None):
    fn_ = _boxes(n_max, frames)
    _check(lib.nms_run_static_batched(_ptr(boxes, "float32", "boxes", 4 * fn_), _ptr(scores, "float32", "scores", fn_),
                                      _ptr(counts, "int32", "counts", int(frames)), int(n_max), int(frames), float(threshold),
                                      _ptr(keep_out, "uint8", "keep_out", fn_), _stream(stream)),
           "nms_run_static_batched")


# ------------------------------------------------------------------ the choices of a decoding step

NMS_TYPE_F32, NMS_TYPE_F16, NMS_TYPE_BF16 = 0, 1, 2
NMS_MAX_FRAMES, NMS_MAX_DRAFTS, NMS_MAX_VOCABULARY, NMS_MAX_SLOTS, NMS_CACHE_MAX_TENSORS = 65535, 1024, 4194304, 1048576, 8
_TYPES = {torch.float32: NMS_TYPE_F32, torch.float16: NMS_TYPE_F16, torch.bfloat16: NMS_TYPE_BF16}


def _beyond_32_bits(**named):
    """ctypes keeps the low 32 bits of a larger number without a word.  For numbers of which one is below 0 or does not fit: the former are the
    library's to refuse."""
    for what, v in named.items():
        if not -2 ** 31 <= v < 2 ** 31:
            raise ValueError(f"{what}: {v} does not fit 32 bits")


def _here(*named):
    """The kernels run on the current device: tensors of another one are refused.  (name, tensor) in turn."""
    device = torch.cuda.current_device()
    for what, t in zip(named[::2], named[1::2]):
        if isinstance(t, _Tensor) and t.is_cuda and t.get_device() != device:
            raise ValueError(f"{what}: tensor lives on {t.device}, the current device is cuda:{device}")


def _strided(t, what):
    if not isinstance(t, _Tensor):
        raise TypeError(f"{what}: expected a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{what}: tensor must live on the GPU")
    return t


def _type_of(t, what):
    if t.dtype not in _TYPES:
        raise TypeError(f"{what}: expected float32, float16 or bfloat16, got {t.dtype}")
    return _TYPES[t.dtype]


def _rows(t, shape, what):
    """(address, stride from row to row) of a tensor whose leading dimensions are `shape` but the last, and whose last holds at least
    shape[-1] neighbouring elements: rows may lie apart, all at one distance."""
    has = tuple(_strided(t, what).shape)
    if has == shape and t.is_contiguous():
        return t.data_ptr(), shape[-1]
    if len(has) != len(shape) or has[:-1] != shape[:-1] or has[-1] < shape[-1]:
        raise ValueError(f"{what}: shape {has}, the call needs {shape}")
    strides = t.stride()
    if shape[-1] > 1 and strides[-1] != 1:
        raise ValueError(f"{what}: the elements of a row must be neighbours")
    row, expect = None, None
    for d in range(len(shape) - 2, -1, -1):
        if shape[d] == 1:
            continue
        if row is None:
            row = expect = strides[d]
        if strides[d] != expect:
            raise ValueError(f"{what}: rows must lie at one distance from each other")
        expect *= shape[d]
    if row is None:
        row = shape[-1]
    if row < shape[-1]:
        raise ValueError(f"{what}: rows must not overlap")
    return t.data_ptr(), row


def nms_verify_workspace_bytes(vocabulary: int, sequences: int) -> int:
    v, s = int(vocabulary), int(sequences)
    if (v | s) >> 31:
        _beyond_32_bits(vocabulary=v, sequences=s)
    return int(lib.nms_verify_workspace_bytes(v, s))


def _verify_arguments(target, draft, drafts, counts, drafts_max, vocabulary, sequences, uniforms, tokens_out, accepted_out, workspace):
    k, v, s = int(drafts_max), int(vocabulary), int(sequences)
    if (k | v | s) >> 31:
        _beyond_32_bits(drafts_max=k, vocabulary=v, sequences=s)
    _here("target", target, "draft", draft, "drafts", drafts, "counts", counts, "uniforms", uniforms, "tokens_out", tokens_out,
          "accepted_out", accepted_out, "workspace", workspace)
    t_at, t_row, d_at, d_row, kind = None, v, None, v, NMS_TYPE_F32
    if 0 <= k <= NMS_MAX_DRAFTS and 1 <= v <= NMS_MAX_VOCABULARY and 1 <= s <= NMS_MAX_FRAMES:  # else the library refuses the sizes, or there is nothing to do
        t_at, t_row = _rows(target, (s, k + 1, v), "target")
        kind = _type_of(target, "target")
        if draft is not None and k > 0:
            d_at, d_row = _rows(draft, (s, k, v), "draft")
            if draft.dtype != target.dtype:
                raise TypeError(f"draft: expected dtype {target.dtype}, got {draft.dtype}")
    need = max(s, 0) * (max(k, 0) + 1)
    w, wb = _ws(workspace)
    return (t_at, t_row, d_at, d_row, kind, _ptr(drafts, "int32", "drafts", max(s, 0) * max(k, 0)), _ptr(counts, "int32", "counts", max(s, 0)),
            k, v, s, _ptr(uniforms, "float32", "uniforms", need), _ptr(tokens_out, "int32", "tokens_out", need),
            _ptr(accepted_out, "int32", "accepted_out", max(s, 0)), w, wb)


def nms_verify_batched(target, draft, drafts, counts, drafts_max, vocabulary, sequences, uniforms, tokens_out, accepted_out, workspace,
                       stream=None):
    """target: [sequences, drafts_max + 1, >= vocabulary]; draft: [sequences, drafts_max, >= vocabulary] of the same dtype, or None.
    Their rows may lie apart (a slice of wider rows), all at one distance."""
    _check(lib.nms_verify_batched(*_verify_arguments(target, draft, drafts, counts, drafts_max, vocabulary, sequences, uniforms,
                                                     tokens_out, accepted_out, workspace), _stream(stream)), "nms_verify_batched")


def nms_cache_moves_max(n_max: int, budget: int) -> int:
    n, b = int(n_max), int(budget)
    if (n | b) >> 31:
        _beyond_32_bits(n_max=n, budget=b)
    return int(lib.nms_cache_moves_max(n, b))


def nms_cache_workspace_bytes(n_max: int, heads: int, sequences: int, budget: int) -> int:
    return int(lib.nms_cache_workspace_bytes(*_cache_sizes(n_max, heads, sequences, budget)[:4]))


def _cache_sizes(n_max, heads, sequences, budget, first=0, recent=0):
    n, h, s, b, f, r = int(n_max), int(heads), int(sequences), int(budget), int(first), int(recent)
    if (n | h | s | b | f | r) >> 31:
        _beyond_32_bits(n_max=n, heads=h, sequences=s, budget=b, first=f, recent=r)
    return n, h, s, b, f, r


def _cache_elements(n_max, heads, sequences):
    """sequences * heads * n_max and sequences; zeros when the library will refuse the sizes anyway."""
    if n_max < 0 or heads < 0 or sequences < 0 or n_max > NMS_MAX_SLOTS or heads * sequences > NMS_MAX_FRAMES:
        return 0, 0
    return sequences * heads * n_max, sequences


def _cache_weights(weights, valid_tokens, heads, sequences):
    """struct nms_cache_weights of a tensor [sequences, heads, group, tokens, columns], or None."""
    if weights is None:
        return None
    shape = tuple(_strided(weights, "weights").shape)
    if len(shape) != 5 or shape[0] != sequences or shape[1] != heads:
        raise ValueError(f"weights: shape {shape}, the call needs ({sequences}, {heads}, group, tokens, columns)")
    at, row = _rows(weights, shape, "weights")
    if (shape[2] | shape[3] | shape[4]) >> 31:
        raise ValueError(f"weights: shape {shape} does not fit 32 bits")
    return NmsCacheWeights(at, row, _type_of(weights, "weights"), shape[2], shape[3], shape[4],
                           _ptr(valid_tokens, "int32", "valid_tokens", sequences))


def _cache_tensor(t, what, n_max, heads, sequences, paged):
    """The fields of struct nms_cache_tensor for a tensor whose rows are whole and lie apart."""
    shape = tuple(_strided(t, what).shape)
    if len(shape) < 3 or shape[1] < heads or (not paged and (shape[0] < sequences or shape[2] < n_max)):
        need = f"({sequences}, {heads}, {n_max}, ...)" if not paged else f"(pages, {heads}, slots of a page, ...)"
        raise ValueError(f"{what}: shape {shape}, the call needs {need}")
    strides, row = t.stride(), 1
    for d in range(len(shape) - 1, 2, -1):
        if shape[d] != 1 and strides[d] != row:
            raise ValueError(f"{what}: the elements of a row must be neighbours")
        row *= shape[d]
    if not t.is_contiguous():
        extent = row
        for stride, size in sorted(zip(strides[:3], shape[:3])):
            if size > 1:
                if stride < extent:
                    raise ValueError(f"{what}: rows must not overlap")
                extent += stride * (size - 1)
    b = t.element_size()
    return t.data_ptr(), row * b, strides[0] * b, strides[1] * b, strides[2] * b


def _cache_tensors(tensors, n_max, heads, sequences, page_table):
    """Array of struct nms_cache_tensor, its length, and struct nms_cache_pages or None."""
    if not tensors:
        return None, 0, None
    structs = (NmsCacheTensor * len(tensors))(*[_cache_tensor(t, f"tensors[{i}]", n_max, heads, sequences, page_table is not None)
                                                for i, t in enumerate(tensors)])
    if page_table is None:
        return structs, len(tensors), None
    count, slots = tensors[0].shape[0], tensors[0].shape[2]
    for i, t in enumerate(tensors):
        if t.shape[0] != count or t.shape[2] != slots:
            raise ValueError(f"tensors[{i}]: pages of the tensors must be as many and as long")
    if not isinstance(page_table, _Tensor) or page_table.dim() != 2 or page_table.shape[0] < sequences:
        raise ValueError(f"page_table: expected a tensor ({sequences}, pages of a sequence)")
    each = -(-max(n_max, 0) // max(slots, 1))
    if page_table.shape[1] < each:
        raise ValueError(f"page_table: {page_table.shape[1]} pages to a sequence, the call needs {each}")
    if (count | slots | page_table.shape[1]) >> 31:
        raise ValueError(f"page_table: {page_table.shape[1]} pages to a sequence, {count} pages of {slots} slots: they do not fit 32 bits")
    return structs, len(tensors), NmsCachePages(_ptr(page_table, "int32", "page_table", 0), page_table.shape[1], slots, count, 0)


def nms_cache_keep_batched(sums, positions, counts, lengths, n_max, heads, sequences, budget, first, recent, keep_out, kept_out, moves_out,
                           workspace, weights=None, valid_tokens=None, stream=None):
    """weights: [sequences, heads, group, tokens, columns], rows at one distance from each other, or None.
    moves_out: at least sequences * heads * (nms_cache_moves_max(n_max, budget) + 1) * 2 elements, or None."""
    n, h, s, b, first, recent = _cache_sizes(n_max, heads, sequences, budget, first, recent)
    _here("sums", sums, "positions", positions, "counts", counts, "lengths", lengths, "keep_out", keep_out, "kept_out", kept_out,
          "moves_out", moves_out, "workspace", workspace, "weights", weights, "valid_tokens", valid_tokens)
    all_, s_ = _cache_elements(n, h, s)
    w, wb = _ws(workspace)
    struct = _cache_weights(weights, valid_tokens, h, s) if all_ else None
    _check(lib.nms_cache_keep_batched(
        _ptr(sums, "float32", "sums", all_), _ptr(positions, "int32", "positions", all_), _ptr(counts, "int32", "counts", s_),
        _ptr(lengths, "int32", "lengths", s_), n, h, s, struct, b, first, recent,
        _ptr(keep_out, "uint8", "keep_out", all_), _ptr(kept_out, "int32", "kept_out", s_),
        _ptr(moves_out, "int32", "moves_out", s_ * h * (max(nms_cache_moves_max(n, b), 0) + 1) * 2 if all_ and moves_out is not None else 0),
        w, wb, _stream(stream)),
        "nms_cache_keep_batched")


def nms_cache_move_batched(moves, n_max, heads, sequences, budget, tensors, page_table=None, stream=None):
    """tensors: up to eight of shape [sequences, heads, n_max, row ...] (any strides whose rows are whole), or with a page table
    ([sequences, pages of a sequence] int32) [pages, heads, slots of a page, row ...]."""
    n, h, s, b, _, _ = _cache_sizes(n_max, heads, sequences, budget)
    tensors = tuple(tensors or ())  # gone over more than once
    _here("moves", moves, "page_table", page_table, *(x for t in tensors for x in ("tensors", t)))
    all_, s_ = _cache_elements(n, h, s)
    structs, many, pages = _cache_tensors(tensors, n, h, s, page_table)
    _check(lib.nms_cache_move_batched(_ptr(moves, "int32", "moves", s_ * h * (max(nms_cache_moves_max(n, b), 0) + 1) * 2 if all_ else 0),
                                      n, h, s, b, structs, many, pages, _stream(stream)), "nms_cache_move_batched")


def _evict_arguments(sums, positions, counts, lengths, n_max, heads, sequences, budget, first, recent, tensors, keep_out, kept_out,
                     workspace, weights, valid_tokens, page_table):
    n, h, s, b, first, recent = _cache_sizes(n_max, heads, sequences, budget, first, recent)
    tensors = tuple(tensors or ())  # gone over more than once
    _here("sums", sums, "positions", positions, "counts", counts, "lengths", lengths, "keep_out", keep_out, "kept_out", kept_out,
          "workspace", workspace, "weights", weights, "valid_tokens", valid_tokens, "page_table", page_table,
          *(x for t in tensors for x in ("tensors", t)))
    all_, s_ = _cache_elements(n, h, s)
    w, wb = _ws(workspace)
    struct = _cache_weights(weights, valid_tokens, h, s) if all_ else None
    structs, many, pages = _cache_tensors(tensors if all_ else (), n, h, s, page_table)
    return (_ptr(sums, "float32", "sums", all_), _ptr(positions, "int32", "positions", all_), _ptr(counts, "int32", "counts", s_),
            _ptr(lengths, "int32", "lengths", s_), n, h, s, struct, b, first, recent, structs, many, pages,
            _ptr(keep_out, "uint8", "keep_out", all_), _ptr(kept_out, "int32", "kept_out", s_), w, wb)


def nms_cache_evict_batched(sums, positions, counts, lengths, n_max, heads, sequences, budget, first, recent, tensors, keep_out, kept_out,
                            workspace, weights=None, valid_tokens=None, page_table=None, stream=None):
    """The whole path: tensors and page_table as nms_cache_move_batched takes them, the rest as nms_cache_keep_batched."""
    _check(lib.nms_cache_evict_batched(*_evict_arguments(sums, positions, counts, lengths, n_max, heads, sequences, budget, first, recent,
                                                         tensors, keep_out, kept_out, workspace, weights, valid_tokens, page_table),
                                       _stream(stream)), "nms_cache_evict_batched")


class _DecodingPlan:
    """A call with its arguments marshalled once, for decoding loops whose buffers stay: each call is then a single foreign call.
    The plan holds references to its tensors; a call uses the stream given here, or the current one of the device that the plan was
    made on; while another one is current it is refused."""

    def __init__(self, entry, args, keepalive, stream):
        self._entry, self._fn, self._args, self._keepalive, self._given = entry, getattr(lib, entry), args, keepalive, stream
        self._current = _current_device if _current_device is not None and torch.cuda.is_initialized() else lambda: torch.cuda.current_device()
        self._device = self._current()

    def __call__(self):
        if self._current() != self._device:
            raise ValueError(f"{self._entry}: the plan was made on cuda:{self._device}, the current device is cuda:{self._current()}")
        status = self._fn(*self._args, _stream(self._given))
        if status != NMS_OK:
            raise NmsError(status, self._entry)


class VerifyPlan(_DecodingPlan):
    """nms_verify_batched, marshalled once."""

    def __init__(self, target, draft, drafts, counts, drafts_max, vocabulary, sequences, uniforms, tokens_out, accepted_out, workspace,
                 stream=None):
        args = (target, draft, drafts, counts, drafts_max, vocabulary, sequences, uniforms, tokens_out, accepted_out, workspace)
        super().__init__("nms_verify_batched", _verify_arguments(*args), args, stream)


class CachePlan(_DecodingPlan):
    """nms_cache_evict_batched, marshalled once."""

    def __init__(self, sums, positions, counts, lengths, n_max, heads, sequences, budget, first, recent, tensors, keep_out, kept_out,
                 workspace, weights=None, valid_tokens=None, page_table=None, stream=None):
        args = (sums, positions, counts, lengths, n_max, heads, sequences, budget, first, recent, tuple(tensors or ()), keep_out, kept_out,
                workspace, weights, valid_tokens, page_table)
        super().__init__("nms_cache_evict_batched", _evict_arguments(*args), args, stream)
