"""ctypes binding of the matrix operators in include/rtopk.h: the orthogonal factor of an update, the master update with
it, linear layers on 8-bit and on 4-bit codes, and what stands between them: dropout and layer normalisation.  Argument
marshalling only, as in binding.py."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from .binding import GRAD_BF16, GRAD_F32, RTopKError, _i64, _vp, load_library

_DTYPES = {torch.float32: GRAD_F32, torch.bfloat16: GRAD_BF16}


def _scratch(what: str, *sizes: int) -> int:
    n = _i64(0)
    rc = getattr(load_library(), what)(*sizes, C.byref(n))
    if rc != 0:
        raise RTopKError(rc, what, load_library().rtopk_status_string(rc).decode())
    return int(n.value)


def orthogonalize_scratch(batch: int, m: int, n: int) -> int:
    """Scratch bytes of :meth:`MatrixContext.orthogonalize` and :meth:`MatrixContext.orthogonal_update`."""
    return _scratch("rtopk_orthogonalize_scratch", batch, m, n)


def coded_scratch(tokens: int, n_out: int, n_in: int) -> int:
    """Scratch bytes of :meth:`MatrixContext.coded_product` and :meth:`MatrixContext.coded_gradients` for up to `tokens` tokens."""
    return _scratch("rtopk_coded_scratch", tokens, n_out, n_in)


def micro_scratch(tokens: int, n_out: int, n_in: int) -> int:
    """Scratch bytes of :meth:`MatrixContext.micro_product` and :meth:`MatrixContext.micro_gradients` for up to `tokens` tokens."""
    return _scratch("rtopk_micro_scratch", tokens, n_out, n_in)


def micro_layout(rows: int, cols: int):
    """(least bytes of a row of 4-bit codes, bytes of the scales) of an array of `rows` rows of `cols` codes."""
    ld, scales = _i64(0), _i64(0)
    rc = load_library().rtopk_micro_layout(rows, cols, C.byref(ld), C.byref(scales))
    if rc != 0:
        raise RTopKError(rc, "rtopk_micro_layout", "invalid argument")
    return int(ld.value), int(scales.value)


def layer_norm_scratch(rows: int, cols: int) -> int:
    """Scratch bytes of :meth:`MatrixContext.layer_norm_gradients` with dgamma or dbeta."""
    return _scratch("rtopk_layer_norm_scratch", rows, cols)


def _dtype(t: torch.Tensor, what: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{what} must be float32 or bfloat16")
    return code


class CodedWeights:
    """The 8-bit codes of an (n_out, n_in) weight matrix and one scale for each output channel: what a master broadcasts.
    ``codes`` is int8 [n_out, ld], ``codes_t`` the same codes transposed (None with ``transposed=False``, for layers that
    take no gradient with respect to their input), ``scales`` float32 [n_out].  Each may be replaced by another tensor of that form, with
    rows of at least the codes' number, contiguous, a multiple of 16 bytes apart; calls use the tensors that are there when they
    are made."""

    def __init__(self, n_out: int, n_in: int, transposed: bool = True, device=None):
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        self._n_out, self._n_in = n_out, n_in
        self.codes = torch.zeros((n_out, -(-n_in // 128) * 128), dtype=torch.int8, device=device)
        self.codes_t = torch.zeros((n_in, -(-n_out // 128) * 128), dtype=torch.int8, device=device) if transposed else None
        self.scales = torch.zeros(n_out, dtype=torch.float32, device=device)

    n_out = property(lambda self: self._n_out)
    n_in = property(lambda self: self._n_in)
    codes = property(lambda self: self._codes)
    codes_t = property(lambda self: self._codes_t)
    scales = property(lambda self: self._scales)

    @codes.setter
    def codes(self, t):
        self._codes = self._checked(t, "codes", self._n_out, self._n_in)

    @codes_t.setter
    def codes_t(self, t):
        self._codes_t = None if t is None else self._checked(t, "codes_t", self._n_in, self._n_out)

    @scales.setter
    def scales(self, t):
        if t.dtype != torch.float32:
            raise TypeError("scales must be float32")
        if t.shape != (self._n_out,) or not t.is_contiguous():
            raise ValueError(f"scales must be contiguous and of shape {(self._n_out,)}")
        self._scales = t

    @staticmethod
    def _checked(t, what, rows, cols):
        if t.dtype != torch.int8:
            raise TypeError(f"{what} must be int8")
        if t.dim() != 2 or t.shape[0] != rows or t.shape[1] < cols or (t.stride(1) != 1 and t.shape[1] > 1):
            raise ValueError(f"{what} must have {rows} contiguous rows of at least {cols} codes")
        return t

    def dense(self) -> torch.Tensor:
        """The values that the codes stand for."""
        return self.codes[:, :self.n_in].float() * self.scales[:, None]


class MicroWeights:
    """The 4-bit codes of an (n_out, n_in) weight matrix with a power of two for each `tile` x 32 of them (`tile` 32, or 1 without the
    transposed codes).  ``codes`` is uint8 [n_out, ld], two codes a byte, ``scales`` uint8 [scale bytes], ``codes_t`` and ``scales_t`` the
    same transposed (None with ``transposed=False``).  Each may be replaced by another tensor of that form; calls use the tensors
    that are there when they are made."""

    def __init__(self, n_out: int, n_in: int, transposed: bool = True, tile: int = 32, device=None):
        if tile not in (1, 32) or (transposed and tile != 32):
            raise ValueError("tile must be 32, or 1 for weights without transposed codes")
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
        self._n_out, self._n_in, self._tile = n_out, n_in, tile

        def arrays(rows, cols):
            ld, scale_bytes = micro_layout(rows, cols)
            return (torch.zeros((rows, -(-ld // 128) * 128), dtype=torch.uint8, device=device),
                    torch.zeros(scale_bytes, dtype=torch.uint8, device=device))
        self.codes, self.scales = arrays(n_out, n_in)
        self.codes_t, self.scales_t = arrays(n_in, n_out) if transposed else (None, None)

    n_out = property(lambda self: self._n_out)
    n_in = property(lambda self: self._n_in)
    tile = property(lambda self: self._tile)
    codes = property(lambda self: self._codes)
    scales = property(lambda self: self._scales)
    codes_t = property(lambda self: self._codes_t)
    scales_t = property(lambda self: self._scales_t)

    @codes.setter
    def codes(self, t):
        self._codes = self._checked_codes(t, "codes", self._n_out, self._n_in)

    @scales.setter
    def scales(self, t):
        self._scales = self._checked_scales(t, "scales", self._n_out, self._n_in)

    @codes_t.setter
    def codes_t(self, t):
        self._codes_t = None if t is None else self._checked_codes(t, "codes_t", self._n_in, self._n_out)

    @scales_t.setter
    def scales_t(self, t):
        self._scales_t = None if t is None else self._checked_scales(t, "scales_t", self._n_in, self._n_out)

    @staticmethod
    def _checked_codes(t, what, rows, cols):
        if t.dtype != torch.uint8:
            raise TypeError(f"{what} must be uint8")
        least = micro_layout(rows, cols)[0]
        if t.dim() != 2 or t.shape[0] != rows or t.shape[1] < least or t.stride(1) != 1:
            raise ValueError(f"{what} must have {rows} contiguous rows of at least {least} bytes")
        return t

    @staticmethod
    def _checked_scales(t, what, rows, cols):
        if t.dtype != torch.uint8:
            raise TypeError(f"{what} must be uint8")
        count = micro_layout(rows, cols)[1]
        if t.shape != (count,) or not t.is_contiguous():
            raise ValueError(f"{what} must be contiguous and of shape {(count,)}")
        return t

    def dense(self) -> torch.Tensor:
        """The values that the codes stand for."""
        byte = self.codes[:, :(self.n_in + 1) // 2].long()
        code = torch.stack((byte & 15, byte >> 4), 2).flatten(1)[:, :self.n_in]
        table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
        value = torch.where(code >= 8, -table[code & 7], table[code & 7])
        r = torch.arange(self.n_out, device=code.device)[:, None]
        b = torch.arange(self.n_in, device=code.device)[None, :] // 32
        pieces = -(-self.n_in // 256) * 2
        scale = self.scales[((r // 128) * pieces + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4].int()
        power = torch.where(scale == 0, 1 << 22, scale << 23).int().view(torch.float32)      # 2^(scale - 127) by its bits
        return torch.where(scale == 255, float("nan"), value * power)


class _MaskStruct(C.Structure):
    _fields_ = [("p", C.c_double), ("seed", C.c_uint64), ("step_ptr", _vp), ("step", C.c_uint32), ("worker", C.c_uint32), ("site", C.c_uint32)]


class Mask:
    """Which elements dropout drops: a share p of them, by (seed, step, worker, site) and their place in the rows; nothing is stored.  `step`
    is a number, or a one-element int32 tensor on the context's device that kernels read when they run (for captured graphs);
    it may be changed from call to call."""

    def __init__(self, p: float, seed: int, step=0, worker: int = 0, site: int = 0):
        if not 0 <= p < 1:
            raise ValueError("p must be at least 0 and less than 1")
        if not 0 <= worker < 65536 or not 0 <= site < 32768:
            raise ValueError("worker must be below 65536 and site below 32768")
        if not 0 <= seed < 1 << 64:
            raise ValueError("seed must be a number of 64 bits")
        self._struct = _MaskStruct(p, seed, None, 0, worker, site)
        self.step = step

    p = property(lambda self: self._struct.p)
    seed = property(lambda self: self._struct.seed)
    worker = property(lambda self: self._struct.worker)
    site = property(lambda self: self._struct.site)
    step = property(lambda self: self._step)

    @step.setter
    def step(self, step):
        if isinstance(step, torch.Tensor):
            if step.dtype != torch.int32 or step.numel() != 1:
                raise ValueError("step must be a number or one int32")
            self._struct.step = 0
        else:
            if not 0 <= step < 1 << 32:
                raise ValueError("step must be a number of 32 bits")
            self._struct.step, self._struct.step_ptr = step, None
        self._step = step

    def __reduce__(self):
        return Mask, (self.p, self.seed, self._step, self.worker, self.site)


class MatrixContext:
    """A context of the matrix operators on one device, with its scratch.  Tensors must live on that device; rows must be
    contiguous (last stride 1), everything else is passed as strides.  Calls go to the current stream; those that share a
    context share its scratch and must follow one another, on one stream or ordered by events.  A graph that captured calls needs
    the context until its last replay."""

    def __init__(self, scratch_bytes: int, device: Optional[int] = None):
        if not torch.cuda.is_available():
            raise RuntimeError("the matrix operators need a CUDA device: there is no CPU fallback")
        self._lib = load_library()
        self._h = None
        self.device = torch.cuda.current_device() if device is None else int(device)
        self._raw_stream = torch._C._cuda_getCurrentRawStream      # the handle alone: a Stream object takes microseconds
        # From torch's allocator, which knows the stream that the scratch was made on; others are made known to it as they come.  That
        # stream may still be using the memory for what it held before, and it clears the library's counters: others wait for it.
        self._scratch = torch.empty(scratch_bytes, dtype=torch.uint8, device=f"cuda:{self.device}") if scratch_bytes > 0 else None
        self._streams = {self._raw_stream(self.device)}
        h = _vp()
        rc = self._lib.rtopk_matrix_create(C.byref(h), self.device, self._scratch.data_ptr() if scratch_bytes > 0 else None,
                                           scratch_bytes, self._stream())
        if rc != 0:
            raise RTopKError(rc, "rtopk_matrix_create", self._lib.rtopk_status_string(rc).decode())
        self._h = h
        self._made = torch.cuda.current_stream(self.device).record_event()

    def _stream(self) -> int:
        s = self._raw_stream(self.device)
        if s not in self._streams:
            stream = torch.cuda.current_stream(self.device)
            if self._scratch is not None:
                self._scratch.record_stream(stream)
            with torch.cuda.device(self.device):
                capturing = torch.cuda.is_current_stream_capturing()
            if not capturing:       # a capture cannot wait for what is outside it; torch.cuda.graph synchronises before
                stream.wait_event(self._made)
                self._streams.add(s)
        return s

    def close(self) -> None:
        if getattr(self, "_h", None):
            self._lib.rtopk_matrix_destroy(self._h)
            self._h = None
            self._scratch = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int, what: str) -> None:
        if rc != 0:
            detail = self._lib.rtopk_status_string(rc).decode()
            if rc == 3:
                detail += f", cudaError {self._lib.rtopk_matrix_last_cuda_error(self._h)}"
            raise RTopKError(rc, what, detail)

    def _on_device(self, t: torch.Tensor, what: str) -> int:
        """The tensor's address; another device's means nothing to the kernels."""
        if t.get_device() != self.device:
            raise ValueError(f"{what} must be on device {self.device}")
        return t.data_ptr()

    def _rows(self, t: torch.Tensor, what: str, shape=None):
        """(pointer, row stride) of a matrix with contiguous rows."""
        sizes = t.shape
        if shape is not None and sizes != shape:
            raise ValueError(f"{what} must have shape {tuple(shape)}, not {tuple(sizes)}")
        ld = sizes[-1]
        if not t.is_contiguous():
            strides = t.stride()
            if strides[-1] != 1 and ld > 1:
                raise ValueError(f"the rows of {what} must be contiguous")
            if sizes[-2] > 1:
                ld = strides[-2]
        if t.get_device() != self.device:
            raise ValueError(f"{what} must be on device {self.device}")
        return t.data_ptr(), ld

    def _batch(self, t: torch.Tensor, what: str, shape=None):
        """(pointer, row stride, matrix stride) of a matrix or a batch of them."""
        if t.dim() not in (2, 3):
            raise ValueError(f"{what} must be a matrix or a batch of matrices")
        p, ld = self._rows(t, what, shape)
        return p, ld, (t.stride(0) if t.dim() == 3 and t.shape[0] > 1 else 0)

    def _codes(self, t: Optional[torch.Tensor]):
        """(pointer, row stride) of an array of codes."""
        return (None, 0) if t is None else (self._on_device(t, "the codes"), t.stride()[0])

    @staticmethod
    def _sizes(t: torch.Tensor):
        return (t.shape[0] if t.dim() == 3 else 1), t.shape[-2], t.shape[-1]

    @staticmethod
    def _coef(coef: Optional[Sequence[Sequence[float]]], steps: int):
        if coef is None:
            return None
        flat = [float(v) for triple in coef for v in triple]
        if len(flat) != 3 * steps:
            raise ValueError("coef must hold one triple for each step")
        return (C.c_float * len(flat))(*flat)

    def orthogonalize(self, src, out, steps=5, coef=None, eps=1e-7) -> None:
        """out <- the orthogonal factor of src ([m, n] or [batch, m, n], float32 or bfloat16) by Newton-Schulz steps."""
        p, ld, stride = self._batch(src, "src")
        po, ldo, strideo = self._batch(out, "out", src.shape)
        rc = self._lib.rtopk_orthogonalize(self._h, p, _dtype(src, "src"), ld, stride, po, _dtype(out, "out"), ldo, strideo,
                                           *self._sizes(src), steps, self._coef(coef, steps), eps, self._stream())
        self._check(rc, "rtopk_orthogonalize")

    def orthogonal_update(self, grad, momentum, weights, eta, mu, nesterov=True, decay=0.0, scale=1.0, steps=5, coef=None,
                          eps=1e-7) -> None:
        """momentum <- mu momentum + grad; weights <- (1 - eta decay) weights - eta scale orth(update), all float32."""
        for t, what in ((grad, "grad"), (momentum, "momentum"), (weights, "weights")):
            if t.dtype != torch.float32:
                raise TypeError(f"{what} must be float32")
        g, ldg, sg = self._batch(grad, "grad")
        v, ldv, sv = self._batch(momentum, "momentum", grad.shape)
        w, ldw, sw = self._batch(weights, "weights", grad.shape)
        rc = self._lib.rtopk_orthogonal_update(self._h, g, ldg, sg, v, ldv, sv, w, ldw, sw, *self._sizes(grad), eta, mu,
                                               1 if nesterov else 0, decay, scale, steps, self._coef(coef, steps), eps,
                                               self._stream())
        self._check(rc, "rtopk_orthogonal_update")

    def code_weights(self, weights, coded: CodedWeights) -> None:
        """coded <- the codes of weights ([n_out, n_in], float32 or bfloat16), one scale for each row."""
        p, ld = self._rows(weights, "weights", (coded.n_out, coded.n_in))
        rc = self._lib.rtopk_code_weights(self._h, p, _dtype(weights, "weights"), ld, coded.n_out, coded.n_in,
                                          *self._codes(coded._codes), *self._codes(coded._codes_t),
                                          self._on_device(coded._scales, "scales"), self._stream())
        self._check(rc, "rtopk_code_weights")

    def coded_product(self, x, coded: CodedWeights, out) -> None:
        """out[t, n] <- x W^T with W as codes and x ([tokens, n_in], float32 or bfloat16) coded for each token."""
        tokens, n_in, n_out, codes = x.shape[0], coded._n_in, coded._n_out, coded._codes
        p, ld = self._rows(x, "x", (tokens, n_in))
        po, ldo = self._rows(out, "out", (tokens, n_out))
        dtype = _DTYPES.get(x.dtype)
        if dtype is None or out.dtype != x.dtype:
            raise TypeError("x must be float32 or bfloat16, and out have its type")
        rc = self._lib.rtopk_coded_product(self._h, p, dtype, ld, self._on_device(codes, "codes"), codes.stride()[0],
                                           self._on_device(coded._scales, "scales"), tokens, n_out, n_in, po, ldo, self._stream())
        if rc:
            self._check(rc, "rtopk_coded_product")

    def coded_gradients(self, dy, x, coded: CodedWeights, dx=None, dw=None) -> None:
        """The gradients of :meth:`coded_product` for dy ([tokens, n_out]): dx like x, dw ([n_out, n_in], float32 or bfloat16).
        Either may be left out; x may be None when dw is."""
        tokens = dy.shape[0]
        py, ldy = self._rows(dy, "dy", (tokens, coded.n_out))
        dt = _dtype(dy, "dy")
        px = ldx = pdx = lddx = pdw = lddw = 0
        wt = GRAD_F32
        if dw is not None:
            if x is None:
                raise ValueError("dw needs x")
            px, ldx = self._rows(x, "x", (tokens, coded.n_in))
            if x.dtype != dy.dtype:
                raise TypeError("x must have the type of dy")
            pdw, lddw = self._rows(dw, "dw", (coded.n_out, coded.n_in))
            wt = _dtype(dw, "dw")
        if dx is not None:
            pdx, lddx = self._rows(dx, "dx", (tokens, coded.n_in))
            if dx.dtype != dy.dtype:
                raise TypeError("dx must have the type of dy")
            if coded._codes_t is None:
                raise ValueError("these weights were made without their transposed codes")
        rc = self._lib.rtopk_coded_gradients(self._h, py, ldy, px, ldx, dt, *self._codes(coded._codes_t),
                                             self._on_device(coded._scales, "scales"), tokens, coded.n_out, coded.n_in, pdx, lddx,
                                             pdw, wt, lddw, self._stream())
        self._check(rc, "rtopk_coded_gradients")

    def micro_weights(self, weights, micro: MicroWeights) -> None:
        """micro <- the 4-bit codes of weights ([n_out, n_in], float32 or bfloat16)."""
        p, ld = self._rows(weights, "weights", (micro.n_out, micro.n_in))
        codes_t, scales_t = micro._codes_t, micro._scales_t
        if (codes_t is None) != (scales_t is None):
            raise ValueError("codes_t and scales_t go together")
        rc = self._lib.rtopk_micro_weights(self._h, p, _dtype(weights, "weights"), ld, micro.n_out, micro.n_in, micro._tile,
                                           *self._codes(micro._codes), self._on_device(micro._scales, "scales"), *self._codes(codes_t),
                                           None if scales_t is None else self._on_device(scales_t, "scales_t"), self._stream())
        self._check(rc, "rtopk_micro_weights")

    def micro_product(self, x, micro: MicroWeights, out) -> None:
        """out[t, n] <- x W^T with W as 4-bit codes and x ([tokens, n_in], float32 or bfloat16) coded in the call."""
        tokens, n_in, n_out, codes = x.shape[0], micro._n_in, micro._n_out, micro._codes
        p, ld = self._rows(x, "x", (tokens, n_in))
        po, ldo = self._rows(out, "out", (tokens, n_out))
        dtype = _DTYPES.get(x.dtype)
        if dtype is None or out.dtype != x.dtype:
            raise TypeError("x must be float32 or bfloat16, and out have its type")
        rc = self._lib.rtopk_micro_product(self._h, p, dtype, ld, self._on_device(codes, "codes"), codes.stride()[0],
                                           self._on_device(micro._scales, "scales"), tokens, n_out, n_in, po, ldo, self._stream())
        if rc:
            self._check(rc, "rtopk_micro_product")

    def micro_gradients(self, dy, x, micro: MicroWeights, dx=None, dw=None) -> None:
        """The gradients of :meth:`micro_product` for dy ([tokens, n_out]): dx like x, dw ([n_out, n_in], float32 or bfloat16).
        Either may be left out; x may be None when dw is."""
        tokens = dy.shape[0]
        py, ldy = self._rows(dy, "dy", (tokens, micro.n_out))
        dt = _dtype(dy, "dy")
        px = ldx = pdx = lddx = pdw = lddw = 0
        wt = GRAD_F32
        codes_t, scales_t = (None, 0), None
        if dw is not None:
            if x is None:
                raise ValueError("dw needs x")
            px, ldx = self._rows(x, "x", (tokens, micro.n_in))
            if x.dtype != dy.dtype:
                raise TypeError("x must have the type of dy")
            pdw, lddw = self._rows(dw, "dw", (micro.n_out, micro.n_in))
            wt = _dtype(dw, "dw")
        if dx is not None:
            pdx, lddx = self._rows(dx, "dx", (tokens, micro.n_in))
            if dx.dtype != dy.dtype:
                raise TypeError("dx must have the type of dy")
            if micro._codes_t is None or micro._scales_t is None:
                raise ValueError("these weights were made without their transposed codes")
            codes_t, scales_t = self._codes(micro._codes_t), self._on_device(micro._scales_t, "scales_t")
        rc = self._lib.rtopk_micro_gradients(self._h, py, ldy, px, ldx, dt, *codes_t, scales_t, tokens, micro.n_out, micro.n_in, pdx,
                                             lddx, pdw, wt, lddw, self._stream())
        self._check(rc, "rtopk_micro_gradients")

    def _mask(self, mask: Optional[Mask]):
        if mask is None:
            return None
        if isinstance(mask._step, torch.Tensor):
            mask._struct.step_ptr = self._on_device(mask._step, "the mask's step")
        return C.byref(mask._struct)

    def _like(self, t, what: str, dtype, shape):
        """(pointer, row stride) of an optional matrix of that type and shape."""
        if t is None:
            return None, 0
        if t.dtype is not dtype:
            raise TypeError(f"{what} must have the other matrices' type")
        if t.shape != shape or not t.is_contiguous():
            return self._rows(t, what, shape)
        if t.get_device() != self.device:
            raise ValueError(f"{what} must be on device {self.device}")
        return t.data_ptr(), shape[1]

    def _vector(self, t, what: str, n: int):
        if t is None:
            return None
        if t.dtype is not torch.float32:
            raise TypeError(f"{what} must be float32")
        if t.numel() != n or t.dim() != 1 or not t.is_contiguous():
            raise ValueError(f"{what} must be contiguous and of shape {(n,)}")
        if t.get_device() != self.device:
            raise ValueError(f"{what} must be on device {self.device}")
        return t.data_ptr()

    @staticmethod
    def _matrix(t, what: str):
        """(shape, torch's type, the library's type) of the matrix that the others are like."""
        shape, dtype = t.shape, t.dtype
        if len(shape) != 2:
            raise ValueError(f"{what} must be a matrix")
        code = _DTYPES.get(dtype)
        if code is None:
            raise TypeError(f"{what} must be float32 or bfloat16")
        return shape, dtype, code

    def dropout(self, x, out, mask: Mask) -> None:
        """out <- x where the mask keeps an element, times 1 / the share that is kept, else 0 ([rows, cols], float32 or bfloat16; out may be
        x).  The gradient is the same call on out's gradient."""
        shape, dtype, code = self._matrix(x, "x")
        p, ld = self._like(x, "x", dtype, shape)
        po, ldo = self._like(out, "out", dtype, shape)
        rc = self._lib.rtopk_dropout(self._h, p, code, ld, *shape, self._mask(mask), po, ldo, self._stream())
        if rc:
            self._check(rc, "rtopk_dropout")

    def layer_norm(self, x, gamma, beta, out, residual=None, total=None, mean=None, rstd=None, eps=1e-5, mask: Optional[Mask] = None) -> None:
        """total <- residual + dropout(x); out <- gamma (total - mean) rstd + beta over each row of [rows, cols] matrices, float32 or bfloat16.
        residual, mask, gamma, beta (float32 [cols]) may be None; total, mean and rstd (float32 [rows]) are written where given, for
        :meth:`layer_norm_gradients`."""
        shape, dtype, code = self._matrix(x, "x")
        rows, cols = shape
        p, ld = self._like(x, "x", dtype, shape)
        pr, ldr = self._like(residual, "residual", dtype, shape)
        po, ldo = self._like(out, "out", dtype, shape)
        pt, ldt = self._like(total, "total", dtype, shape)
        rc = self._lib.rtopk_layer_norm(self._h, p, ld, pr, ldr, code, rows, cols, self._vector(gamma, "gamma", cols),
                                        self._vector(beta, "beta", cols), eps, self._mask(mask), po, ldo, pt, ldt,
                                        self._vector(mean, "mean", rows), self._vector(rstd, "rstd", rows), self._stream())
        if rc:
            self._check(rc, "rtopk_layer_norm")

    def layer_norm_gradients(self, dy, total, mean, rstd, gamma, dresidual=None, dgamma=None, dbeta=None, dtotal=None, dx=None,
                             mask: Optional[Mask] = None) -> None:
        """The gradients of :meth:`layer_norm` for dy (of out) and dtotal (of total, where it is used elsewhere; may be None): dresidual (without
        a mask also that of x), dx with a mask, dgamma and dbeta (float32 [cols]).  total, mean and rstd are the forward call's;
        without residual and mask, total is its x."""
        shape, dtype, code = self._matrix(dy, "dy")
        if (mask is None) != (dx is None):
            raise ValueError("dx goes with a mask: without one it is dresidual")
        rows, cols = shape
        p, ld = self._like(dy, "dy", dtype, shape)
        pt, ldt = self._like(total, "total", dtype, shape)
        pa, lda = self._like(dtotal, "dtotal", dtype, shape)
        pr, ldr = self._like(dresidual, "dresidual", dtype, shape)
        px, ldx = self._like(dx, "dx", dtype, shape)
        rc = self._lib.rtopk_layer_norm_gradients(self._h, p, ld, pt, ldt, pa, lda, code, rows, cols, self._vector(mean, "mean", rows),
                                                  self._vector(rstd, "rstd", rows), self._vector(gamma, "gamma", cols), self._mask(mask), pr, ldr,
                                                  px, ldx, self._vector(dgamma, "dgamma", cols), self._vector(dbeta, "dbeta", cols), self._stream())
        if rc:
            self._check(rc, "rtopk_layer_norm_gradients")

    def set_option(self, option: int, value: int) -> None:
        self._check(self._lib.rtopk_matrix_set_option(self._h, option, value), "rtopk_matrix_set_option")

    def poll_status(self) -> None:
        self._check(self._lib.rtopk_matrix_poll_status(self._h, self._stream()), "rtopk_matrix_poll_status")

    def launch_count(self) -> int:
        n = C.c_uint64(0)
        self._check(self._lib.rtopk_matrix_get_launch_count(self._h, C.byref(n)), "rtopk_matrix_get_launch_count")
        return int(n.value)
