"""Paged 4-bit key/value cache (include/ivfpq_kv.h): page tables from request lengths, append,
page selection, attention.  As in `binding`, this module marshals arguments: torch supplies device memory
and the current stream, every step runs in the HIP kernels, and there is no fallback.

One step of a server that decodes `requests` requests:

    step = kv.plan(past_lens, new_lens, table, free_pages, free_state, max_tokens=T)
    cache.append(k, v, step.slots)                              # k, v [T][kv_heads][head_dim]
    pages = cache.select(q, step, 64)                           # optional: 64 pages a token and kv head
    out, lse = cache.attention(q, step, pages=pages, max_new=1)     # q [T][heads][head_dim]
    past_lens, free_state = step.kv_lens, step.free_state

One that checks drafted tokens, a tree of them a request (its first token is the last one that is certain):

    step = kv.plan(past_lens, new_lens, table, free_pages, free_state, max_tokens=T)
    tree = kv.tree(parents, step, max_nodes=N)                  # what each sees of the others, and its position
    q, k = rotary(q, k, tree.positions)                         # rotary = kv.Rotary(frequencies, axes), once
    cache.append(k, v, step.slots)
    out, lse = cache.tree_attention(q, step, tree)              # these three in each layer
    kept = kv.keep(caches, step, tree, drafted, picked, free_pages, step.free_state)   # all layers' caches
    past_lens, free_state = kept.lens, kept.free_state
"""
from __future__ import annotations

import ctypes
from fractions import Fraction
from typing import Optional, Sequence, Tuple

import torch

from .binding import IvfpqError, _check, _dev, load_library  # noqa: F401

PAGE = 64
MAX_REQUESTS, MAX_SELECT, MAX_NODES, MAX_AXES = 65536, 1024, 1024, 8
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}

# every symbol include/ivfpq_kv.h declares
SYMBOLS = [
    "ivfpq_kv_page_bytes", "ivfpq_kv_plan", "ivfpq_kv_append", "ivfpq_kv_select_workspace_bytes", "ivfpq_kv_select",
    "ivfpq_kv_attention_workspace_bytes", "ivfpq_kv_attention", "ivfpq_kv_rotate", "ivfpq_kv_tree_plan",
    "ivfpq_kv_tree_attention_workspace_bytes", "ivfpq_kv_tree_attention", "ivfpq_kv_keep", "ivfpq_kv_read",
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


class _Rotary(ctypes.Structure):
    _fields_ = [("head_dim", _i32), ("turned", _i32), ("neighbours", _i32), ("dtype", _i32), ("axes", _i32), ("phases", _vp),
                ("axis", _vp)]


class _Tree(ctypes.Structure):
    _fields_ = [("max_nodes", _i32), ("window", _i32), ("masks", _vp), ("positions", _vp)]


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
        tp = ctypes.POINTER(_Tree)
        lib.ivfpq_kv_rotate.argtypes = [ctypes.POINTER(_Rotary), _Rows, _i32, _Rows, _i32, _vp, _i64, _i64, _Rows, _Rows, _vp]
        lib.ivfpq_kv_tree_plan.argtypes = [sp, _vp, tp, _vp]
        lib.ivfpq_kv_tree_attention_workspace_bytes.argtypes = [cp, sp, ap, tp]
        lib.ivfpq_kv_tree_attention_workspace_bytes.restype = _sz
        lib.ivfpq_kv_tree_attention.argtypes = [cp, sp, ap, tp, _vp, _sz, _vp]
        lib.ivfpq_kv_keep.argtypes = [_vp, _i32, sp, tp, _vp, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp]
        lib.ivfpq_kv_read.argtypes = [cp, _vp, _i64, _Rows, _Rows, _vp]
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
    try:
        if t.dtype is dtype and t.shape == shape and t.get_device() == device:
            ts, hs, cs = t.stride()
            if cs == 1:
                return _Rows(t.data_ptr(), ts, hs)
    except AttributeError:
        pass
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


def _needs_gradient() -> None:
    """For tensors whose gradient a result without a graph would lose, or that a graph holds and a result would overwrite."""
    if torch.is_grad_enabled():
        raise ValueError("there is no backward pass: tensors that need a gradient are taken under torch.no_grad() or detached")


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


class Tree:
    """What `tree` leaves for attention and `keep`: masks [T][ceil(max_nodes / 64)] int64 (bit j % 64 of word j / 64: the request's
    j-th new token is seen), positions [T] int32 (-1 in rows without a token)."""

    def __init__(self, masks: torch.Tensor, positions: torch.Tensor, max_nodes: int, window: int = 0):
        if not 1 <= max_nodes <= MAX_NODES:
            raise ValueError(f"max_nodes = {max_nodes} outside [1, {MAX_NODES}]")
        if not 0 <= window < 1 << 31:
            raise ValueError(f"window = {window} outside [0, 2^31)")
        T = masks.shape[0]
        self._checked = dev = _dev(masks, torch.int64, (T, (max_nodes + 63) // 64), what="masks").device.index
        _dev(positions, torch.int32, (T,), dev, "positions")
        self.masks, self.positions, self.max_nodes, self.window, self.max_tokens = masks, positions, max_nodes, window, T
        self._c = _Tree(max_nodes, window, masks.data_ptr(), positions.data_ptr())
        self._ref, self._held = ctypes.byref(self._c), (masks, positions)

    @classmethod
    def empty(cls, max_tokens: int, max_nodes: int, window: int = 0, device=None) -> "Tree":
        """Buffers for the trees of a step, to be filled by `tree(..., out=tree)`."""
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        return cls(torch.empty(max_tokens, (max_nodes + 63) // 64, dtype=torch.int64, device=device),
                   torch.empty(max_tokens, dtype=torch.int32, device=device), max_nodes, window)


def _fits(step: Step, tree: Tree) -> None:
    if tree.max_tokens != step.max_tokens or tree._checked != step._checked:
        raise ValueError(f"tree: {tree.max_tokens} rows on cuda:{tree._checked}, the step has {step.max_tokens} on cuda:{step._checked}")


def tree(parents: torch.Tensor, step: Step, max_nodes: Optional[int] = None, window: Optional[int] = None, out: Optional[Tree] = None) -> Tree:
    """What drafted tokens see of each other, and their positions (`ivfpq_kv_tree_plan`).  parents [T] int32: the number, within
    its request, of the token that each hangs on; -1: none.  max_nodes: no request has more new tokens (T unless given, 1024 at
    most).  It decides how wide masks are and how `tree_attention` cuts its work, not what is computed: with several requests give the
    largest tree's, as T takes many small trees for a few large ones, which is slower.  window: positions that a token sees, its own
    among them (0: all).  Both are those of `out` where that is given."""
    if out is None:
        out = Tree.empty(step.max_tokens, min(max(step.max_tokens, 1), MAX_NODES) if max_nodes is None else max_nodes, window or 0,
                         step.table.device)
    elif (max_nodes is not None and max_nodes != out.max_nodes) or (window is not None and window != out.window):
        raise ValueError(f"tree: out was made for max_nodes = {out.max_nodes} and window = {out.window}")
    _fits(step, out)
    dev = step._checked
    _launch(dev, _lib().ivfpq_kv_tree_plan, step._ref, _ptr(parents, torch.int32, (step.max_tokens,), dev, "parents"), out._ref)
    return out


# 2 pi 2^200, rounded: frequencies are divided by it as whole numbers
_TWO_PI = 10096689509235987743946820282484873672429286842977325943070736


class Rotary:
    """Rotary positions (`ivfpq_kv_rotate`).  frequencies: radians a position, one for each pair of channels (their number a
    multiple of 8: the first 2 len(frequencies) channels are turned); axes: which axis of the position turns each pair (all the first,
    unless given), such as time, height and width; neighbours: pairs are channels 2 i and 2 i + 1 instead of i and i + len(frequencies).
    To be made once for a model: its table is computed on the host in whole numbers (half a millisecond) and depends on no position."""

    def __init__(self, frequencies: Sequence[float], axes: Optional[Sequence[int]] = None, neighbours: bool = False, device=None):
        frequencies = [float(f) for f in frequencies]
        axes = [0] * len(frequencies) if axes is None else [int(a) for a in axes]
        if not frequencies or len(frequencies) % 8 or len(frequencies) > 128:
            raise ValueError(f"{len(frequencies)} frequencies: a multiple of 8 up to 128 is needed")
        if len(axes) != len(frequencies) or not all(0 <= a < MAX_AXES for a in axes):
            raise ValueError(f"axes: one of 0 .. {MAX_AXES - 1} is needed for each of the {len(frequencies)} frequencies")
        if not all(abs(f) < float("inf") for f in frequencies):
            raise ValueError("frequencies must be finite")
        turns = [round(Fraction(f) * (1 << 264) / _TWO_PI) % (1 << 64) for f in frequencies]
        device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
        self._phases = torch.tensor([t - (1 << 64) if t >> 63 else t for t in turns], dtype=torch.int64, device=device)
        self._axis = torch.tensor(axes, dtype=torch.int32, device=device)
        self._refs = {}  # the call's description for each head_dim and type
        self.device, self.axes, self.turned, self.neighbours = self._phases.device.index, max(axes) + 1, 2 * len(turns), bool(neighbours)

    def __call__(self, q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor,
                 out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """q [T][heads][head_dim] and k [T][kv_heads][head_dim] turned by positions [axes][T] int32 ([T]: the same on every axis);
        a token whose first position is negative is left out: its rows are not written.  out: two tensors for the results, q and k
        themselves among them; no other overlap.  There is no backward pass: tensors that need a gradient are refused."""
        heads, kv_heads, dev = _heads_of(q), _heads_of(k), self.device
        if q.requires_grad or k.requires_grad:
            _needs_gradient()
        T, _, D = q.shape
        dtype = q.dtype
        if dtype not in _DTYPES:
            raise ValueError(f"q must be of torch.bfloat16 or torch.float16, not {dtype}")
        shape_q, shape_k = (T, heads, D), (T, kv_heads, D)
        qr, kr = _rows(q, dtype, shape_q, dev, "q"), _rows(k, dtype, shape_k, dev, "k")
        one = isinstance(positions, torch.Tensor) and positions.dim() == 1
        at = _ptr(positions, torch.int32, (T,) if one else (self.axes, T), dev, "positions")
        if out is None:
            out = torch.empty(shape_q, dtype=dtype, device=q.device), torch.empty(shape_k, dtype=dtype, device=q.device)
        to_q, to_k = _rows(out[0], dtype, shape_q, dev, "out q"), _rows(out[1], dtype, shape_k, dev, "out k")
        if out[0].requires_grad or out[1].requires_grad:
            _needs_gradient()
        ref = self._refs.get((D, dtype))
        if ref is None:
            c = _Rotary(_int32(D, "head_dim"), self.turned, self.neighbours, _DTYPES[dtype], self.axes, self._phases.data_ptr(), self._axis.data_ptr())
            ref = self._refs[D, dtype] = ctypes.byref(c)
        _launch(dev, _lib().ivfpq_kv_rotate, ref, qr, heads, kr, kv_heads, at, 0 if one else T, T, to_q, to_k)
        return out[0], out[1]


class Kept:
    """What `keep` leaves: lens [R] int32, the tokens that each request holds from now on; rows [T] int32, of request r from
    q_start[r] on the rows that stay, -1 behind them; free_state [3] int64 of the next plan."""

    def __init__(self, lens: torch.Tensor, rows: torch.Tensor, free_state: torch.Tensor):
        R, T = lens.shape[0], rows.shape[0]
        self._checked = dev = _dev(free_state, torch.int64, (3,), what="free_state").device.index
        _dev(lens, torch.int32, (R,), dev, "lens")
        _dev(rows, torch.int32, (T,), dev, "rows")
        self.lens, self.rows, self.free_state = lens, rows, free_state
        counts = torch.empty(R, dtype=torch.int32, device=lens.device)  # room for keep
        self._shape = R, T
        self._at = free_state.data_ptr(), lens.data_ptr(), rows.data_ptr(), counts.data_ptr()
        self._held = lens, rows, free_state, counts

    @classmethod
    def empty(cls, step: Step) -> "Kept":
        """Buffers for `keep(..., out=kept)` after steps of this size."""
        def new(n, dtype=torch.int32):
            return torch.empty(n, dtype=dtype, device=step.table.device)
        return cls(new(step.kv_lens.shape[0]), new(step.max_tokens), new(3, torch.int64))


def keep(caches: Sequence["KvCache"], step: Step, tree: Tree, drafted: torch.Tensor, picked: torch.Tensor, free_pages: torch.Tensor,
         free_state: torch.Tensor, out: Optional[Kept] = None) -> Kept:
    """What stays of a step's drafted tokens (`ivfpq_kv_keep`): of every request its first new token and the longest path behind
    it whose tokens are those that the model picked.  (With masks of the caller's own: the deepest token that sees only tokens that agree, and
    what it sees; none of a request's where there is no such token, as in a block that sees all of itself and is refused.)  They move
    together in all caches (of one shape), the boxes of their pages are made again, pages behind them go back to the ring.  tree: the
    step's, without a window; drafted, picked [T] int32: the tokens, and what the model picks behind each; free_state:
    `step.free_state`.  Once per step."""
    caches = list(caches)
    _fits(step, tree)
    dev, T = step._checked, step.max_tokens
    if not all(c.device == dev for c in caches):
        raise ValueError(f"caches: not all on cuda:{dev}, where the step is")
    if out is None:
        out = Kept.empty(step)
    elif out._shape != (step.kv_lens.shape[0], T) or out._checked != dev:
        raise ValueError(f"keep: out was made for steps of {out._shape} requests and rows on cuda:{out._checked}")
    state_out, lens, rows, counts = out._at
    ring = _ptr(free_pages, torch.int32, free_pages.shape[:1], dev, "free_pages")
    _launch(dev, _lib().ivfpq_kv_keep, (_Cache * len(caches))(*[c._c for c in caches]), len(caches), step._ref, tree._ref,
            _ptr(drafted, torch.int32, (T,), dev, "drafted"), _ptr(picked, torch.int32, (T,), dev, "picked"), ring, free_pages.shape[0],
            _ptr(free_state, torch.int64, (3,), dev, "free_state"), state_out, lens, rows, counts)
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
        (out as q, rows that do not overlap; lse [T][heads] fp32), without a graph: there is no backward pass."""
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

    def tree_attention_workspace(self, step: Step, heads: int, tree: Tree) -> torch.Tensor:
        _fits(step, tree)
        args = _Attention(heads=heads, max_new=1)
        return self._workspace(_lib().ivfpq_kv_tree_attention_workspace_bytes(self._ref, self._step(step), ctypes.byref(args), tree._ref))

    def tree_attention(self, q: torch.Tensor, step: Step, tree: Tree, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                       lse: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None):
        """Drafted tokens' attention over the cache (`ivfpq_kv_tree_attention`): over what their requests held before the step (with a
        window of the tree the last of it) and over the new tokens that their masks name.  q [T][heads][head_dim]; scale: head_dim
        ** -0.5 unless given.  There is no backward pass: tensors that need a gradient are refused.  Returns (out as q, rows that do not
        overlap; lse [T][heads] fp32)."""
        T, heads, dev, dtype = step.max_tokens, _heads_of(q), self.device, self.dtype
        if q.requires_grad:
            _needs_gradient()
        _fits(step, tree)
        shape = (T, heads, self.head_dim)
        qr = _rows(q, dtype, shape, dev, "q")
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=q.device)
        to = _rows(out, dtype, shape, dev, "out")
        if lse is None:
            lse = torch.empty((T, heads), dtype=torch.float32, device=q.device)
        to_lse = _ptr(lse, torch.float32, (T, heads), dev, "lse")
        if out.requires_grad or lse.requires_grad:
            _needs_gradient()
        ws = self.tree_attention_workspace(step, heads, tree) if workspace is None else workspace
        size = ws.shape[0]
        args = _Attention(qr, heads, 1, self.head_dim ** -0.5 if scale is None else scale, 0, None, 0, to.data, to.token_stride,
                          to.head_stride, to_lse)
        _launch(dev, _lib().ivfpq_kv_tree_attention, self._ref, self._step(step), ctypes.byref(args), tree._ref,
                _ptr(ws, torch.uint8, (size,), dev, "workspace"), size)
        return out, lse

    def read(self, slots: torch.Tensor, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """Held keys and values at slots [T] int64 as rows [T][kv_heads][head_dim] (`ivfpq_kv_read`); 0 for slots outside the cache."""
        shape = (slots.shape[0], self.kv_heads, self.head_dim)
        dtype, dev = self.dtype, self.device
        at = _ptr(slots, torch.int64, shape[:1], dev, "slots")
        if out is None:
            out = torch.empty(shape, dtype=dtype, device=slots.device), torch.empty(shape, dtype=dtype, device=slots.device)
        kr, vr = _rows(out[0], dtype, shape, dev, "out k"), _rows(out[1], dtype, shape, dev, "out v")
        _launch(dev, _lib().ivfpq_kv_read, self._ref, at, shape[0], kr, vr)
        return out[0], out[1]
