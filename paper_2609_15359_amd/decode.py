"""One decode step of a decoder: the block tables of the blocks that placement
counts, the KV cache that they address (held in 4 bits), attention over it, and
the verification of drafted tokens.  Thin front end of the library calls of the
same names, like the rest of the binding; shapes, types and strides are checked
here on the host."""
from __future__ import annotations

from dataclasses import dataclass
from functools import lru_cache

import torch

from . import MapsError, _check, _dev, _stream, check_errors, library, new_error_word

MAX_STEP_REQUESTS = 8192
MAX_CACHE_BLOCK = 256
MAX_DRAFTS = 64
_TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}

# A step makes these calls once a layer, on kernels of a few microseconds: the checks take the quick way where a
# tensor is as it should be, pointers go to the library as numbers, and the stream is asked for by its device's index.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _dense(t, dtype, name):
    """_dev, without its cost for a plain tensor that passes."""
    if type(t) is torch.Tensor and t.is_cuda and t.dtype is dtype and t.is_contiguous():
        return t
    return _dev(t, dtype, name)


def _at(t):
    return None if t is None else t.data_ptr()


def _current(t):
    """The current stream of t's device."""
    return _raw_stream(t.get_device()) if _raw_stream is not None else _stream(t.device)


def _apart(written, others):
    """Raises unless every dense tensor of `written` shares no byte with the others of it and with `others`."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), w)
                   for ts, w in ((written, True), (others, False)) for t in ts if t.numel())
    last = last_written = 0                  # ends of the spans so far
    for start, end, w in spans:
        if start < (last if w else last_written):
            raise MapsError("out's arrays must not overlap each other or the ones that the call reads")
        last = max(last, end)
        if w:
            last_written = max(last_written, end)


@lru_cache(maxsize=4096)
def _size(name, device, *sizes):
    """A size query of the library, which depends on its arguments and, if `device` is not None, on the current device's
    compute units."""
    return int(getattr(library(), name)(*sizes))


def _current_device():
    return torch.cuda.current_device() if torch.cuda.is_initialized() else -1


def _scratch(nbytes, t, given):
    """`given` where it is large enough, else a new workspace beside t."""
    if given is not None and _dense(given, torch.uint8, "workspace").numel() >= nbytes:
        return given
    return t.new_empty(max(int(nbytes), 1), dtype=torch.uint8)


# ---------------------------------------------------------------------------
# 5. block tables and slots
# ---------------------------------------------------------------------------

@dataclass
class BlockStep:
    """What one step of the block tables gives (maps_block_step)."""
    slots: torch.Tensor       # [T] int64: cache slot of each new token, -1 where refused or past the last
    tok_off: torch.Tensor     # [B + 1] int64: the new tokens of request slot b
    lens: torch.Tensor        # [B] int32, tokens after the step
    held: torch.Tensor        # [B] int32, blocks after the step
    ring_pos: torch.Tensor    # [2] int32, the ring's front and count after the step
    granted: torch.Tensor     # [B] uint8, 0: refused, its new tokens have no slots (kv_attend takes this array)
    dev_err: torch.Tensor


def block_step(grow, table, held, lens, ring, ring_pos, block_size: int, total: int, done=None, dev_err=None,
               out: BlockStep | None = None) -> BlockStep:
    """Grows B request slots by `grow` tokens: blocks from the ring of free
    blocks, the slot of each of the `total` new tokens; `done` slots give their
    blocks back first.  table and ring are updated in place; held, lens and
    ring_pos are read, their new values are the result's (out: a result of an
    earlier call to write into, not one that this call reads)."""
    _dense(grow, torch.int32, "grow")
    B, N, T = grow.numel(), _dense(ring, torch.int32, "ring").numel(), int(total)
    _dense(table, torch.int32, "table")
    if table.dim() != 2 or table.shape[0] != B:
        raise MapsError(f"table must be [B, max_blocks] with B = {B} (got {tuple(table.shape)})")
    for name, t, n in (("held", held, B), ("lens", lens, B), ("ring_pos", ring_pos, 2)):
        if _dense(t, torch.int32, name).numel() != n:
            raise MapsError(f"{name} must have {n} entries")
    if done is not None and _dense(done, torch.uint8, "done").numel() != B:
        raise MapsError(f"done must have {B} entries")
    if T < 0:
        raise MapsError("total must not be negative")
    err = new_error_word(grow.device) if dev_err is None else dev_err
    if out is None:
        new = grow.new_empty
        out = BlockStep(slots=new(T, dtype=torch.int64), tok_off=new(B + 1, dtype=torch.int64), lens=new(B), held=new(B),
                        ring_pos=new(2), granted=new(B, dtype=torch.uint8), dev_err=err)
    else:
        given = (("slots", torch.int64, T), ("tok_off", torch.int64, B + 1), ("lens", torch.int32, B),
                 ("held", torch.int32, B), ("ring_pos", torch.int32, 2), ("granted", torch.uint8, B))
        for name, dtype, n in given:
            t = _dense(getattr(out, name), dtype, "out." + name)
            if t.numel() != n:
                raise MapsError(f"out was made for another step's sizes: {name} must have {n} entries")
            if t.get_device() != grow.get_device():
                raise MapsError(f"out.{name} must be on {grow.device} (got {t.device})")
        _apart([getattr(out, name) for name, _, _ in given], [grow, lens, held, table, ring, ring_pos, err] +
               ([] if done is None else [done]))
        out.dev_err = err
    st = library().maps_block_step(B, table.shape[1], int(block_size), N, _at(done), _at(grow), _at(lens),
                                   _at(held), _at(table), _at(ring), _at(ring_pos), _at(out.lens),
                                   _at(out.held), _at(out.ring_pos), _at(out.tok_off), _at(out.slots), T,
                                   _at(out.granted), _at(err), _current(grow))
    _check(st, "maps_block_step")
    return out


class BlockTables:
    """The block tables of one decoder's request slots from step to step: B
    slots of at most max_blocks blocks each, over num_blocks blocks of
    block_size tokens, all free at first."""

    def __init__(self, B: int, max_blocks: int, num_blocks: int, block_size: int, device="cuda"):
        i32 = dict(dtype=torch.int32, device=device)
        self.block_size = int(block_size)
        self.table = torch.full((B, max_blocks), -1, **i32)
        self.ring = torch.arange(num_blocks, **i32)
        self.ring_pos = torch.tensor([0, num_blocks], **i32)
        self.lens, self.held = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.dev_err = new_error_word(self.table.device)

    def step(self, grow, total: int, done=None) -> BlockStep:
        """One maps_block_step; the tables go on from its result."""
        r = block_step(grow, self.table, self.held, self.lens, self.ring, self.ring_pos, self.block_size, total, done,
                       self.dev_err)
        self.lens, self.held, self.ring_pos = r.lens, r.held, r.ring_pos
        return r


# ---------------------------------------------------------------------------
# 6. the KV cache in 4 bits, and attention over it
# ---------------------------------------------------------------------------

@dataclass
class KVCache:
    """A paged KV cache of 4-bit values: data is uint8 [num_blocks, heads,
    page bytes] (layout in include/maps.h)."""
    data: torch.Tensor
    block_size: int
    dim: int

    def __post_init__(self):
        _dense(self.data, torch.uint8, "data")
        if self.data.dim() != 3 or self.data.shape[2] != self.page_bytes(self.block_size, self.dim):
            raise MapsError(f"data must be [num_blocks, heads, page bytes] for block_size = {self.block_size}, "
                            f"dim = {self.dim} (got {tuple(self.data.shape)})")

    @staticmethod
    def page_bytes(block_size: int, dim: int) -> int:
        """Bytes of one block of one KV head; block_size is a power of two in
        [16, 256], dim 64, 128 or 256."""
        n = _size("maps_kv_page_bytes", None, int(block_size), int(dim))
        if n == 0:
            raise MapsError(f"no page of block_size = {block_size}, dim = {dim}: block_size is a power of two in "
                            f"[16, {MAX_CACHE_BLOCK}], dim 64, 128 or 256")
        return n

    @classmethod
    def bytes_per_token(cls, heads: int, dim: int) -> int:
        """KV bytes of one token in one layer, for capacity_tokens."""
        return heads * cls.page_bytes(16, dim) // 16

    @classmethod
    def empty(cls, num_blocks: int, heads: int, dim: int, block_size: int, device="cuda") -> "KVCache":
        """A cache whose contents are unspecified until tokens are appended."""
        n = cls.page_bytes(block_size, dim)
        return cls(torch.empty((num_blocks, heads, n), dtype=torch.uint8, device=device), int(block_size), int(dim))

    @property
    def num_blocks(self) -> int:
        return self.data.shape[0]

    @property
    def heads(self) -> int:
        return self.data.shape[1]


def _rows(t, dtypes, shape, name):
    """A device tensor of the given shape (None: any size) whose last axis is dense; the other strides are free."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if not t.is_cuda:
        raise MapsError(f"{name} must be a device tensor (got {t.device})")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} must be one of {', '.join(map(str, dtypes))} (got {t.dtype})")
    if t.shape != shape and (t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape))):
        raise MapsError(f"{name} must be {list(shape)} (got {tuple(t.shape)})")
    if t.stride(-1) != 1 and t.shape[-1] > 1 and t.numel():
        raise MapsError(f"{name}'s last axis must be dense")
    return t


def kv_append(cache: KVCache, k, v, slots, dev_err=None):
    """Quantises T tokens' keys and values ([T, heads, dim]) into the cache at
    `slots` (negative: skipped; the others must differ).  Returns dev_err."""
    T = _dense(slots, torch.int64, "slots").numel()
    _rows(k, tuple(_TYPES), (T, cache.heads, cache.dim), "k")
    _rows(v, (k.dtype,), (T, cache.heads, cache.dim), "v")
    err = new_error_word(slots.device) if dev_err is None else dev_err
    st = library().maps_kv_append(_at(cache.data), cache.num_blocks, cache.block_size, cache.heads, cache.dim,
                                  _at(k), _at(v), _TYPES[k.dtype], T, k.stride(0), k.stride(1), v.stride(0),
                                  v.stride(1), _at(slots), _at(err), _current(slots))
    _check(st, "maps_kv_append")
    return err


def kv_read(cache: KVCache, slots, dtype=torch.bfloat16, dev_err=None, out=None):
    """The keys and values that the cache holds at `slots`, as two dense
    [T, heads, dim] tensors (zeros at negative slots)."""
    T = _dense(slots, torch.int64, "slots").numel()
    if dtype not in _TYPES:
        raise TypeError(f"dtype must be one of {', '.join(map(str, _TYPES))} (got {dtype})")
    shape = (T, cache.heads, cache.dim)
    if out is None:
        out = (slots.new_empty(shape, dtype=dtype), slots.new_empty(shape, dtype=dtype))
    for t in out:
        if _dense(t, dtype, "out").shape != shape:
            raise MapsError(f"out must be two tensors {list(shape)}")
    err = new_error_word(slots.device) if dev_err is None else dev_err
    st = library().maps_kv_read(_at(cache.data), cache.num_blocks, cache.block_size, cache.heads, cache.dim,
                                _at(slots), T, _at(out[0]), _at(out[1]), _TYPES[dtype], _at(err), _current(slots))
    _check(st, "maps_kv_read")
    if dev_err is None:
        check_errors(err)
    return out


def kv_attend_workspace_bytes(B: int, T: int, q_heads: int, heads: int, dim: int, max_q: int) -> int:
    """Bytes that kv_attend's workspace needs on the current device."""
    return _size("maps_kv_attend_workspace_size", _current_device(), int(B), int(T), int(q_heads), int(heads), int(dim),
                 int(max_q))


def kv_attend(cache: KVCache, q, table, lens, tok_off, max_q: int, scale: float, window: int = 0,
              want_lse: bool = False, dev_err=None, workspace=None, out=None, lse=None, granted=None):
    """Attention of the step's query tokens q [T, q_heads, dim] (request b's
    are tok_off[b] .. tok_off[b+1]-1, the last of its lens[b] tokens) over the
    cache, causal, with a sliding window of `window` positions if that is not
    0.  granted: the step's, for a pool that can be short: a refused request's
    new tokens are not in the cache, and its rows get out = 0, lse = -infinity.
    Returns (out [T, q_heads, dim], lse [T, q_heads] or None)."""
    _rows(q, (torch.bfloat16, torch.float16), (None, None, cache.dim), "q")
    T, Hq, dim = q.shape
    heads = cache.heads
    B = _dense(lens, torch.int32, "lens").numel()
    _dense(table, torch.int32, "table")
    if table.dim() != 2 or table.shape[0] != B:
        raise MapsError(f"table must be [B, max_blocks] with B = {B} (got {tuple(table.shape)})")
    if _dense(tok_off, torch.int64, "tok_off").numel() != B + 1:
        raise MapsError(f"tok_off must have {B + 1} entries")
    if granted is not None:
        if _dense(granted, torch.uint8, "granted").numel() != B:
            raise MapsError(f"granted must have {B} entries")
        lens = lens * (granted != 0)
    if out is None:
        out = q.new_empty((T, Hq, dim))
    elif _dense(out, q.dtype, "out").shape != q.shape:
        raise MapsError(f"out must be {list(q.shape)}")
    if lse is None:
        lse = q.new_empty((T, Hq), dtype=torch.float32) if want_lse else None
    elif _dense(lse, torch.float32, "lse").shape != (T, Hq):
        raise MapsError(f"lse must be {[T, Hq]}")
    err = new_error_word(q.device) if dev_err is None else dev_err
    ws = _scratch(kv_attend_workspace_bytes(B, T, Hq, heads, dim, max_q), q, workspace)
    st = library().maps_kv_attend(_at(cache.data), cache.num_blocks, cache.block_size, heads, dim, _at(q),
                            _TYPES[q.dtype], T, Hq, q.stride(0), q.stride(1), _at(table), B, table.shape[1],
                            _at(lens), _at(tok_off), int(max_q), float(scale), int(window), _at(out), _at(lse),
                            _at(err), _at(ws), ws.numel(), _current(q))
    _check(st, "maps_kv_attend")
    if dev_err is None:
        check_errors(err)
    return out, lse


# ---------------------------------------------------------------------------
# 7. verification of drafted tokens
# ---------------------------------------------------------------------------

def verify_drafts(target, draft_tokens, n_draft, u, noise, draft=None, dev_err=None, workspace=None, out=None):
    """Verifies each request's drafted tokens ([B, K]) against the target's
    probabilities ([B, K + 1, V]); draft: the probabilities that they were
    drawn from ([B, K, V]), None where they were not drawn.  u [B, K] uniform,
    noise [B, V] exponential.  Returns (tokens [B, K + 1]: the accepted drafts,
    the next token, then -1; accepted [B])."""
    B, K = _dense(draft_tokens, torch.int32, "draft_tokens").shape
    _rows(target, tuple(_TYPES), (B, K + 1, None), "target")
    V = target.shape[2]
    if draft is not None:
        _rows(draft, (target.dtype,), (B, K, V), "draft")
    if _dense(n_draft, torch.int32, "n_draft").numel() != B:
        raise MapsError(f"n_draft must have {B} entries")
    if _dense(u, torch.float32, "u").shape != (B, K):
        raise MapsError(f"u must be {[B, K]}")
    _rows(noise, (torch.float32,), (B, V), "noise")
    tokens, accepted = out if out is not None else (n_draft.new_empty((B, K + 1)), n_draft.new_empty(B))
    if _dense(tokens, torch.int32, "tokens").shape != (B, K + 1) or _dense(accepted, torch.int32, "accepted").numel() != B:
        raise MapsError("out must be tokens [B, K + 1] and accepted [B]")
    if B == 0:
        return tokens, accepted
    err = new_error_word(target.device) if dev_err is None else dev_err
    ws = _scratch(_size("maps_verify_drafts_workspace_size", None, B, V), target, workspace)
    st = library().maps_verify_drafts(B, K, V, _at(target), target.stride(0), target.stride(1), _at(draft),
                                0 if draft is None else draft.stride(0), 0 if draft is None else draft.stride(1),
                                _TYPES[target.dtype], _at(draft_tokens), _at(n_draft), _at(u), _at(noise),
                                noise.stride(0), _at(tokens), _at(accepted), _at(err), _at(ws), ws.numel(),
                                _current(target))
    _check(st, "maps_verify_drafts")
    if dev_err is None:
        check_errors(err)
    return tokens, accepted
