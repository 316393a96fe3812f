"""Paged 4-bit key/value cache (include/ivfpq_kv.h): page tables from request lengths, append,
page selection, attention.  As in `binding`, this module marshals arguments: torch supplies device memory
and the current stream, every step runs in the HIP kernels, and there is no fallback.

One step of a server that decodes `requests` requests:

    step = kv.plan(past_lens, new_lens, table, free_pages, free_state, max_tokens=T)
    cache.append(k, v, step.slots)                              # k, v [T][kv_heads][head_dim]
    pages = cache.select(q, step, 64)                           # optional: 64 pages a token and kv head
    out, lse = cache.attention(q, step, pages=pages, max_new=1)     # q [T][heads][head_dim]
    past_lens, free_state = step.kv_lens, step.free_state
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from .binding import IvfpqError, _check, _dev, load_library  # noqa: F401

PAGE = 64
MAX_REQUESTS, MAX_SELECT = 65536, 1024
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}

# every symbol include/ivfpq_kv.h declares
SYMBOLS = [
    "ivfpq_kv_page_bytes", "ivfpq_kv_plan", "ivfpq_kv_append", "ivfpq_kv_select_workspace_bytes", "ivfpq_kv_select",
    "ivfpq_kv_attention_workspace_bytes", "ivfpq_kv_attention",
]

_vp, _i64, _i32, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t


class _Cache(ctypes.Structure):
    _fields_ = [("n_pages", _i64), ("kv_heads", _i32), ("head_dim", _i32), ("dtype", _i32), ("pages", _vp), ("boxes", _vp)]


class _Step(ctypes.Structure):
    _fields_ = [("requests", _i32), ("max_tokens", _i32), ("table_width", _i32), ("table", _vp), ("kv_lens", _vp),
                ("q_start", _vp), ("slots", _vp), ("token_req", _vp), ("positions", _vp), ("counts", _vp)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", _vp), ("token_stride", _i64), ("head_stride", _i64)]


class _Attention(ctypes.Structure):
    _fields_ = [("q", _Rows), ("heads", _i32), ("max_new", _i32), ("scale", ctypes.c_float), ("window", _i32),
                ("selected", _vp), ("n_select", _i32), ("out", _vp), ("out_token_stride", _i64), ("out_head_stride", _i64),
                ("lse", _vp)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = load_library()
        cp, sp, ap = ctypes.POINTER(_Cache), ctypes.POINTER(_Step), ctypes.POINTER(_Attention)
        lib.ivfpq_kv_page_bytes.argtypes = [_i32, _i32]
        lib.ivfpq_kv_page_bytes.restype = _sz
        lib.ivfpq_kv_plan.argtypes = [sp, _vp, _vp, _vp, _i64, _vp, _vp, _vp]
        lib.ivfpq_kv_append.argtypes = [cp, _Rows, _Rows, _vp, _i64, _vp, _vp, _vp]
        lib.ivfpq_kv_select_workspace_bytes.argtypes = [cp, sp, _i32]
        lib.ivfpq_kv_select_workspace_bytes.restype = _sz
        lib.ivfpq_kv_select.argtypes = [cp, sp, _Rows, _i32, _i32, _i32, _i32, _vp, _vp, _sz, _vp]
        lib.ivfpq_kv_attention_workspace_bytes.argtypes = [cp, sp, ap]
        lib.ivfpq_kv_attention_workspace_bytes.restype = _sz
        lib.ivfpq_kv_attention.argtypes = [cp, sp, ap, _vp, _sz, _vp]
        _ready = lib
    return _ready


# The checks below run several times in every call of a decode loop, where the host is what
# costs: one comparison each where everything fits, the full check with its message where it does not.


def _ptr(t: torch.Tensor, dtype, shape, device: int, what: str) -> int:
    """Address of a contiguous tensor of this dtype, shape (None: any extent) and device."""
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    return _dev(t, dtype, shape, device, what).data_ptr()


def _rows(t: torch.Tensor, dtype, shape, device: int, what: str) -> _Rows:
    """Rows [tokens][heads][head_dim] that the kernels may read or write where they are: any strides
    of tokens and heads that keep rows on 16 bytes, channels contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype is not dtype:
        raise ValueError(f"{what}: expected a CUDA tensor of {dtype}, got {getattr(t, 'dtype', type(t))} on "
                         f"{getattr(t, 'device', 'the host')}")
    if t.get_device() != device:
        raise ValueError(f"{what}: on {t.device}, the cache lives on cuda:{device}")
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)} does not match {tuple(shape)}")
    ts, hs, cs = t.stride()
    if cs != 1 and t.numel():  # (strides of nothing are arbitrary)
        raise ValueError(f"{what}: the channels must be contiguous, their stride is {cs}")
    return _Rows(t.data_ptr() or None, ts, hs)


def _int32(x: int, what: str) -> int:
    """A number that the library's 32 bits hold; ctypes would drop what is above them."""
    if not -(1 << 31) <= x < 1 << 31:
        raise ValueError(f"{what} = {x} does not fit 32 bits")
    return x


def _heads_of(q: torch.Tensor) -> int:
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q: expected a tensor [tokens][heads][head_dim]")
    return q.shape[1]


_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _launch(device: int, call, *args) -> None:
    """`call` with the stream that is current on the tensors' device, which is made the current one: the library launches there."""
    if _current_device() == device:
        status = call(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            status = call(*args, _raw_stream(device))
    if status:
        _check(status)


class Step:
    """What `plan` leaves for the other calls; every field is a device tensor.

    kv_lens [R] int32, q_start [R + 1] int32, table [R][W] int32 (the caller's), slots [T] int64,
    requests [T] int32, positions [T] int32 (-1 in rows without a token), free_state [3] int64: the
    ring's counters after the step and how many pages were missing."""

    def __init__(self, kv_lens, q_start, table, slots, requests, positions, free_state):
        self.kv_lens, self.q_start, self.table, self.slots = kv_lens, q_start, table, slots
        self.requests, self.positions, self.free_state = requests, positions, free_state
        R, T = kv_lens.shape[0], slots.shape[0]
        self._checked = _dev(table, torch.int32, (R, None), what="table").device.index
        dev = self._checked
        _dev(kv_lens, torch.int32, (R,), dev, "kv_lens")
        _dev(q_start, torch.int32, (R + 1,), dev, "q_start")
        _dev(slots, torch.int64, (T,), dev, "slots")
        _dev(requests, torch.int32, (T,), dev, "requests")
        _dev(positions, torch.int32, (T,), dev, "positions")
        _dev(free_state, torch.int64, (3,), dev, "free_state")
        self.max_tokens = T
        counts = torch.empty(2 * R, dtype=torch.int32, device=table.device)  # room for plan
        self._c = _Step(R, T, table.shape[1], table.data_ptr(), kv_lens.data_ptr(), q_start.data_ptr(), slots.data_ptr(),
                        requests.data_ptr(), positions.data_ptr(), counts.data_ptr() or None)
        self._ref, self._state = ctypes.byref(self._c), free_state.data_ptr()
        self._held = (kv_lens, q_start, table, slots, requests, positions, free_state, counts)  # what the addresses above belong to

    @classmethod
    def empty(cls, requests: int, max_tokens: int, table: torch.Tensor) -> "Step":
        """Buffers for a step, to be filled by `plan(..., out=step)`."""
        def new(n, dtype=torch.int32):
            return torch.empty(n, dtype=dtype, device=table.device)
        return cls(new(requests), new(requests + 1), table, new(max_tokens, torch.int64), new(max_tokens), new(max_tokens),
                   new(3, torch.int64))


def plan(past_lens: torch.Tensor, new_lens: torch.Tensor, table: torch.Tensor, free_pages: torch.Tensor,
         free_state: torch.Tensor, max_tokens: Optional[int] = None, out: Optional[Step] = None) -> Step:
    """Page tables and slot maps of a step (`ivfpq_kv_plan`).  past_lens, new_lens [R] int32 (new < 0: the request
    ends); table [R][W] and free_pages [capacity] int32 are updated in place; free_state [3] int64.
    `free_state[2]` of the result says how many pages were missing: their tokens are not stored."""
    if out is None:
        if max_tokens is None:
            raise ValueError("plan: max_tokens, the most new tokens of the step, is needed without out")
        table = _dev(table, torch.int32, (None, None), what="table")
        out = Step.empty(table.shape[0], int(max_tokens), table)
    elif max_tokens is not None and max_tokens != out.max_tokens:
        raise ValueError(f"plan: out has {out.max_tokens} rows, max_tokens is {max_tokens}")
    c, dev = out._c, out._checked
    R = c.requests
    if _ptr(table, torch.int32, (R, c.table_width), dev, "table") != (c.table or 0):
        raise ValueError("plan: out was made for another table")
    ring = _ptr(free_pages, torch.int32, free_pages.shape[:1], dev, "free_pages")
    _launch(dev, _lib().ivfpq_kv_plan, out._ref, _ptr(past_lens, torch.int32, (R,), dev, "past_lens"),
            _ptr(new_lens, torch.int32, (R,), dev, "new_lens"), ring, free_pages.shape[0],
            _ptr(free_state, torch.int64, (3,), dev, "free_state"), out._state)
    return out


class KvCache:
    """Device memory of a paged 4-bit cache: `pages` (uint8, the layout of include/ivfpq_kv.h) and `boxes`
    [n_pages][kv_heads][2][head_dim] bf16, the smallest and largest key value of each channel of a page."""

    def __init__(self, n_pages: int, kv_heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16, device=None):
        if dtype not in _DTYPES:
            raise ValueError(f"dtype must be torch.bfloat16 or torch.float16, not {dtype}")
        size = _lib().ivfpq_kv_page_bytes(_int32(kv_heads, "kv_heads"), _int32(head_dim, "head_dim"))
        if size == 0:
            raise ValueError(f"kv_heads = {kv_heads} outside [1, 1024] or head_dim = {head_dim} not 64, 96, 128 or 256")
        if not 1 <= n_pages <= 1 << 25:
            raise ValueError(f"n_pages = {n_pages} outside [1, 2^25]")
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self.n_pages, self.kv_heads, self.head_dim, self.dtype = n_pages, kv_heads, head_dim, dtype
        self.pages = torch.zeros(n_pages, size, dtype=torch.uint8, device=device)
        self.boxes = torch.zeros(n_pages, kv_heads, 2, head_dim, dtype=torch.bfloat16, device=device)
        self.device = self.pages.device.index
        self._c = _Cache(n_pages, kv_heads, head_dim, _DTYPES[dtype], self.pages.data_ptr(), self.boxes.data_ptr())
        self._held = (self.pages, self.boxes)
        self._ref = ctypes.byref(self._c)

    def free_ring(self) -> Tuple[torch.Tensor, torch.Tensor]:
        """(free_pages, free_state) of a cache whose pages are all free."""
        dev = self.pages.device
        return (torch.arange(self.n_pages, dtype=torch.int32, device=dev),
                torch.tensor([0, self.n_pages, 0], dtype=torch.int64, device=dev))

    def append(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
               rounded: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> None:
        """Rounds k, v [T][kv_heads][head_dim] into the pages at slots [T] int64; `rounded`: two tensors of that shape
        for the values as they are held."""
        shape = (slots.shape[0], self.kv_heads, self.head_dim)
        dtype, dev = self.dtype, self.device
        kr, vr = _rows(k, dtype, shape, dev, "k"), _rows(v, dtype, shape, dev, "v")
        at = _ptr(slots, torch.int64, shape[:1], dev, "slots")
        to_k = to_v = None
        if rounded is not None:
            to_k, to_v = _ptr(rounded[0], dtype, shape, dev, "rounded k"), _ptr(rounded[1], dtype, shape, dev, "rounded v")
        _launch(dev, _lib().ivfpq_kv_append, self._ref, kr, vr, at, shape[0], to_k, to_v)

    def _step(self, step: Step):
        if step._checked != self.device:
            raise ValueError(f"step: on cuda:{step._checked}, the cache lives on cuda:{self.device}")
        return step._ref

    def _workspace(self, need: int) -> torch.Tensor:
        return torch.empty(max(need, 1), dtype=torch.uint8, device=self.pages.device)

    def select_workspace(self, step: Step, heads: int) -> torch.Tensor:
        return self._workspace(_lib().ivfpq_kv_select_workspace_bytes(self._ref, self._step(step), heads))

    def select(self, q: torch.Tensor, step: Step, n_pages: int, sinks: int = 1, recent: int = 1,
               out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The n_pages table columns that each token and kv head looks at, ascending, -1 behind them
        (`ivfpq_kv_select`): [T][kv_heads][n_pages] int32.  q [T][heads][head_dim]."""
        T, heads, dev = step.max_tokens, _heads_of(q), self.device
        qr = _rows(q, self.dtype, (T, heads, self.head_dim), dev, "q")
        _int32(n_pages, "n_pages")
        if out is None:
            out = torch.empty((T, self.kv_heads, max(n_pages, 0)), dtype=torch.int32, device=q.device)
        to = _ptr(out, torch.int32, (T, self.kv_heads, max(n_pages, 0)), dev, "out")
        sinks, recent = _int32(sinks, "sinks"), _int32(recent, "recent")
        ws = self.select_workspace(step, heads) if workspace is None else workspace
        size = ws.shape[0]
        _launch(dev, _lib().ivfpq_kv_select, self._ref, self._step(step), qr, heads, n_pages, sinks, recent, to,
                _ptr(ws, torch.uint8, (size,), dev, "workspace"), size)
        return out

    def attention_workspace(self, step: Step, heads: int, max_new: Optional[int] = None, n_select: int = 0) -> torch.Tensor:
        max_new = step.max_tokens if max_new is None else _int32(max_new, "max_new")
        args = _Attention(heads=heads, max_new=max_new, n_select=_int32(n_select, "n_select"))
        return self._workspace(_lib().ivfpq_kv_attention_workspace_bytes(self._ref, self._step(step), ctypes.byref(args)))

    def attention(self, q: torch.Tensor, step: Step, scale: Optional[float] = None, window: int = 0,
                  pages: Optional[torch.Tensor] = None, max_new: Optional[int] = None, out: Optional[torch.Tensor] = None,
                  lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        """The new tokens' attention over the cache (`ivfpq_kv_attention`), the new tokens among the keys.
        q [T][heads][head_dim]; scale: head_dim ** -0.5 unless given; window: tokens seen, the token itself among
        them (0: all); pages: [T][kv_heads][n] int32 as from `select`, in any order, none twice (its tokens would count
        twice); max_new: no request has more new tokens (T unless given).  It decides how the work is cut and not what is
        computed: without it a batch that decodes goes through the kernel of chunks, which takes longer.  Returns
        (out as q, rows that do not overlap; lse [T][heads] fp32)."""
        T, heads, dev, dtype = step.max_tokens, _heads_of(q), self.device, self.dtype
        shape = (T, heads, self.head_dim)
        qr = _rows(q, dtype, shape, dev, "q")
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=q.device)
        to = _rows(out, dtype, shape, dev, "out")
        if lse is None:
            lse = torch.empty((T, heads), dtype=torch.float32, device=q.device)
        to_lse = _ptr(lse, torch.float32, (T, heads), dev, "lse")
        n_select, lists = 0, None
        if pages is not None:
            n_select = pages.shape[-1]
            lists = _ptr(pages, torch.int32, (T, self.kv_heads, n_select), dev, "pages") or None
            if n_select < 1:
                raise ValueError("pages: at least one page for a token and kv head")
        if max_new is None:
            max_new = max(T, 1)
        if not (0 <= window < 1 << 31 and 0 < max_new < 1 << 31):
            _int32(window, "window"), _int32(max_new, "max_new")
        ws = self.attention_workspace(step, heads, max_new, n_select) if workspace is None else workspace
        size = ws.shape[0]
        args = _Attention(qr, heads, max_new, self.head_dim ** -0.5 if scale is None else scale, window, lists, n_select,
                          to.data, to.token_stride, to.head_stride, to_lse)
        _launch(dev, _lib().ivfpq_kv_attention, self._ref, self._step(step), ctypes.byref(args),
                _ptr(ws, torch.uint8, (size,), dev, "workspace"), size)
        return out, lse
