"""Python binding of the ps_soft C ABI (include/ps_soft.h): argument checks and marshalling only.

Softmax cross entropy over a whole item table, distillation from a teacher's top scores (both
with the gradients of both tables) and each row's best items run in the HIP kernels of
``libps_mf.so``; this module checks torch tensors and passes their pointers.  ``PsSoft`` wraps a
handle; the library is required: importing this module raises if it is not built.

Tensors live on one GPU.  Calls run on torch's current stream of that GPU, like torch's own
operators, and return without waiting for it.
"""
from __future__ import annotations

import ctypes

import torch

from paper_1410_8043_amd import ps_mf as _mf

LIB_PATH = _mf.LIB_PATH
OK, EINVAL, ENOMEM, EDEVICE, ESTATE = 0, -1, -2, -3, -4
F32, BF16, F16 = 0, 1, 2
OPT_DEVICE, OPT_SPLITS, OPT_SEARCH = 1, 2, 3
TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
MAX_TOP = 256

SYMBOLS = ("ps_soft_create", "ps_soft_set_option", "ps_soft_set_stream", "ps_soft_reserve", "ps_soft_xent", "ps_soft_distill",
           "ps_soft_top", "ps_soft_last_error", "ps_soft_destroy")


def _bind():
    lib = ctypes.CDLL(LIB_PATH)
    i64, i32, f32, vp = ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_void_p
    sig = {
        "ps_soft_create": [i64, i32, i32, ctypes.POINTER(vp)],
        "ps_soft_set_option": [vp, i32, i64],
        "ps_soft_set_stream": [vp, vp],
        "ps_soft_reserve": [vp, i64, i64, i32],
        "ps_soft_xent": [vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, vp, vp, vp, vp, i64, vp, i64],
        "ps_soft_distill": [vp, i64, vp, i64, vp, i64, i32, vp, vp, i64, f32, vp, vp, vp, vp, vp, i64, vp, i64],
        "ps_soft_top": [vp, i64, vp, i64, vp, i64, i32, vp, vp, i64, vp, vp, i64],
    }
    for name, args in sig.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = ctypes.c_int
    lib.ps_soft_last_error.argtypes = [vp]
    lib.ps_soft_last_error.restype = ctypes.c_char_p
    lib.ps_soft_destroy.argtypes = [vp]
    lib.ps_soft_destroy.restype = None
    return lib


_lib = _bind()


class PsSoftError(RuntimeError):
    def __init__(self, func, code, msg):
        super().__init__(f"{func} failed ({code}): {msg}")
        self.code = code


def _check(h, func, rc):
    if rc != OK:
        msg = _lib.ps_soft_last_error(h) if h else b""
        raise PsSoftError(func, rc, (msg or b"").decode(errors="replace"))


def ps_soft_create(items, K, type):
    h = ctypes.c_void_p()
    _check(None, "ps_soft_create", _lib.ps_soft_create(int(items), int(K), int(type), ctypes.byref(h)))
    return h


def _ptr(t):
    return None if t is None else t.data_ptr()


class PsSoft:
    """A handle for tables of ``items`` rows of K numbers: its calls share a workspace that grows to the
    largest call (``reserve`` grows it ahead, as a call that will be captured into a graph needs).

    ``splits`` forces the number of pieces that the reduced axis is cut into (0: by the sizes), ``search`` the form of
    ``top`` (0: all scores in 64 bits, 1: candidates first, None: by the sizes; same results).
    """

    def __init__(self, items, K, dtype=torch.float32, *, device=None, splits=0, search=None):
        if dtype not in TYPES:
            raise ValueError(f"dtype must be one of {', '.join(map(str, TYPES))}, not {dtype}")
        self.items, self.K, self.dtype = int(items), int(K), dtype
        self.device = None
        self._stream = None
        self.h = ps_soft_create(items, K, TYPES[dtype])
        try:
            if splits:
                _check(self.h, "ps_soft_set_option", _lib.ps_soft_set_option(self.h, OPT_SPLITS, int(splits)))
            if search is not None:
                _check(self.h, "ps_soft_set_option", _lib.ps_soft_set_option(self.h, OPT_SEARCH, int(search)))
            if device is not None:
                self._open(torch.device("cuda", device) if isinstance(device, int) else torch.device(device))
        except Exception:
            self.close()
            raise

    def close(self):
        if getattr(self, "h", None):
            _lib.ps_soft_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.close()

    # ---- checks
    def _open(self, device):
        if not self.h:
            raise ValueError("the handle is closed")
        if device.type != "cuda":
            raise ValueError(f"tensors must be on a GPU, not on {device}")
        index = torch.cuda.current_device() if device.index is None else device.index
        if self.device is None:
            _check(self.h, "ps_soft_set_option", _lib.ps_soft_set_option(self.h, OPT_DEVICE, index))
            self.device = torch.device("cuda", index)
        elif self.device.index != index:
            raise ValueError(f"the handle is on {self.device}, the tensor on {device}")

    def _table(self, name, t, rows):
        if not isinstance(t, torch.Tensor) or t.dim() != 2 or t.shape[1] != self.K or (rows is not None and t.shape[0] != rows):
            raise ValueError(f"{name} must be a tensor of {'n' if rows is None else rows} x {self.K}")
        if t.dtype != self.dtype:
            raise ValueError(f"{name} must be {self.dtype}, not {t.dtype}")
        self._open(t.device)
        if t.shape[0] > 0 and self.K > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}'s rows must be contiguous")
        if t.shape[0] > 1 and t.stride(0) < self.K:
            raise ValueError(f"{name}'s rows overlap (stride {t.stride(0)})")
        return t, max(self.K, t.stride(0)) if t.shape[0] > 1 else self.K

    def _list(self, name, t, dtype, shape):
        if t is None:
            return None
        if not isinstance(t, torch.Tensor) or t.dtype != dtype:
            raise ValueError(f"{name} must be a tensor of {dtype}")
        self._open(t.device)
        if t.dim() != len(shape) or any(s is not None and s != d for s, d in zip(shape, t.shape)):
            raise ValueError(f"{name} must have shape {tuple('any' if s is None else s for s in shape)}, not {tuple(t.shape)}")
        return t if t.is_contiguous() else t.contiguous()

    @staticmethod
    def _no_graph(**tensors):
        """Refuse what autograd would take for a constant without a word."""
        if torch.is_grad_enabled():
            for name, t in tensors.items():
                if isinstance(t, torch.Tensor) and t.requires_grad:
                    raise ValueError(f"{name} requires a gradient, which autograd does not get from this call: pass {name}.detach(), or call "
                                     "under torch.no_grad(), and use the gradients that the call returns")

    def _on_stream(self):
        s = torch.cuda.current_stream(self.device).cuda_stream
        if s != self._stream:
            _check(self.h, "ps_soft_set_stream", _lib.ps_soft_set_stream(self.h, s))
            self._stream = s

    def _outputs(self, n, grad):
        new = lambda *shape, dtype: torch.empty(shape, dtype=dtype, device=self.device)  # noqa: E731
        loss, lse = new(n, dtype=torch.float32), new(n, dtype=torch.float32)
        if isinstance(grad, bool):
            grad = "XW" if grad else ""
        if not isinstance(grad, str) or set(grad) - set("XW"):
            raise ValueError("grad must be True, False, 'X', 'W' or 'XW'")
        dX = new(n, self.K, dtype=self.dtype) if "X" in grad else None
        dW = new(self.items, self.K, dtype=self.dtype) if "W" in grad else None
        return loss, lse, dX, dW, bool(grad)

    # ---- calls
    def reserve(self, n, entries, top=0):
        """Grow the workspace to what calls of up to n rows, ``entries`` targets or exclusions and ``top`` items
        per row need."""
        if self.device is None:
            self._open(torch.device("cuda"))
        self._on_stream()
        _check(self.h, "ps_soft_reserve", _lib.ps_soft_reserve(self.h, int(n), int(entries), int(top)))

    def xent(self, X, W, item, *, row_ptr=None, value=None, weight=None, grad=True):
        """Softmax cross entropy of the rows' target items.

        ``item`` int32: one target per row [n], or with ``row_ptr`` int64 [n + 1] the entries of row i
        at row_ptr[i] .. row_ptr[i + 1], with ``value`` fp32 (None: 1) each; an item < 0 is none.  ``weight`` fp32
        [n] (None: 1) weights the rows in the gradients; rows without target or of weight 0 are masked.
        Returns (loss [n], lse [n]) and with ``grad`` (True, or 'X' / 'W' for one of them) also dX, dW.  Autograd does not
        see the call: tensors that require gradients are refused unless it is off.
        """
        self._no_graph(X=X, W=W, value=value, weight=weight)
        X, ldx = self._table("X", X, None)
        W, ldw = self._table("W", W, self.items)
        n = X.shape[0]
        row_ptr = self._list("row_ptr", row_ptr, torch.int64, (n + 1,))
        if item is None:
            raise ValueError("item is required")
        item = self._list("item", item, torch.int32, (n if row_ptr is None else None,))
        value = self._list("value", value, torch.float32, (item.shape[0],))
        weight = self._list("weight", weight, torch.float32, (n,))
        loss, lse, dX, dW, any_grad = self._outputs(n, grad)
        self._on_stream()
        _check(self.h, "ps_soft_xent",
               _lib.ps_soft_xent(self.h, n, _ptr(X), ldx, _ptr(W), ldw, _ptr(row_ptr), _ptr(item), _ptr(value), item.shape[0],
                                 _ptr(weight), _ptr(loss), _ptr(lse), _ptr(dX), self.K, _ptr(dW), self.K))
        return (loss, lse, dX, dW) if any_grad else (loss, lse)

    def distill(self, X, W, item, score, *, tau=1.0, tlse=None, weight=None, grad=True):
        """Divergence of the softmax at temperature ``tau`` from a teacher's.

        ``item`` int32 and ``score`` fp32 [n, k]: the teacher's items and its scores of them; an item < 0 or a
        score of -inf is no entry.  ``tlse`` fp32 [n]: the teacher's log-sum-exp of score / tau over all its items (None:
        its softmax is over the k).  ``weight``, ``grad``, the returned values and what is said of autograd are those of ``xent``.
        """
        self._no_graph(X=X, W=W, score=score, tlse=tlse, weight=weight)
        X, ldx = self._table("X", X, None)
        W, ldw = self._table("W", W, self.items)
        n = X.shape[0]
        if item is None or score is None:
            raise ValueError("item and score are required")
        item = self._list("item", item, torch.int32, (n, None))
        k = item.shape[1]
        if k < 1:
            raise ValueError("the teacher's lists are empty")
        score = self._list("score", score, torch.float32, (n, k))
        tlse = self._list("tlse", tlse, torch.float32, (n,))
        weight = self._list("weight", weight, torch.float32, (n,))
        loss, lse, dX, dW, any_grad = self._outputs(n, grad)
        self._on_stream()
        _check(self.h, "ps_soft_distill",
               _lib.ps_soft_distill(self.h, n, _ptr(X), ldx, _ptr(W), ldw, k, _ptr(item), _ptr(score), k, float(tau), _ptr(tlse),
                                    _ptr(weight), _ptr(loss), _ptr(lse), _ptr(dX), self.K, _ptr(dW), self.K))
        return (loss, lse, dX, dW) if any_grad else (loss, lse)

    def top(self, X, W, k, *, row_ptr=None, item=None):
        """The k items of the largest scores of each row, in order, without those that the row excludes (entries
        row_ptr[i] .. row_ptr[i + 1] of ``item``).  Returns (items int32 [n, k], scores fp32 [n, k]); item -1 and
        score -inf where fewer are left.  The scores carry no gradient."""
        X, ldx = self._table("X", X, None)
        W, ldw = self._table("W", W, self.items)
        n = X.shape[0]
        if (row_ptr is None) != (item is None):
            raise ValueError("row_ptr and item come together")
        k = int(k)
        if not 1 <= k <= MAX_TOP:
            raise ValueError(f"k must be in [1, {MAX_TOP}]")
        row_ptr = self._list("row_ptr", row_ptr, torch.int64, (n + 1,))
        item = self._list("item", item, torch.int32, (None,))
        best = torch.empty((n, k), dtype=torch.int32, device=self.device)
        score = torch.empty((n, k), dtype=torch.float32, device=self.device)
        self._on_stream()
        _check(self.h, "ps_soft_top",
               _lib.ps_soft_top(self.h, n, _ptr(X), ldx, _ptr(W), ldw, k, _ptr(row_ptr), _ptr(item),
                                0 if item is None else item.shape[0], _ptr(best), _ptr(score), k))
        return best, score
