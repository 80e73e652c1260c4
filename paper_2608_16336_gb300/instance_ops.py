"""The operators of one instance's iteration on the GPU (include/mtsim_ops.h).

The simulation charges an iteration a base time plus so much a prefill token
and a decode request; the paper's simulator takes such times from operators
profiled on a GPU (Sec. 2.5, 4.1).  These are the operators to profile, over
the same kind of block-paged cache: ``rotary``, ``latent_append``,
``latent_decode``, ``latent_prefill`` and ``sample``.  ``instance.py`` runs
them together as an instance would and fits the three times.

Each function takes CUDA tensors of the current device and queues its kernels
on the current stream of PyTorch.  Nothing synchronises; scratch memory comes
from PyTorch's allocator on that stream.  Arguments are checked here (shape,
type, place, alignment: ``ValueError`` or ``TypeError``) and again by the
library (``mtsim.SimError``).  Values on the device are bounded by the kernels
as the header states.  The operators are forward only: a tensor that asks for a
gradient is refused while gradients are enabled, one with a forward-mode tangent
while those are (the gradient of ``rotary`` is ``rotary`` with
``inverse=True``).  What a call writes into a tensor of the caller's counts as a
change in place: autograd refuses a backward pass that saved it before.
"""
from __future__ import annotations

import ctypes
import math
from struct import Struct

import torch
from torch.autograd import forward_ad

from . import mtsim

TYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
LAYOUTS = {"interleaved": 0, "half": 1}
MAX_ROT, MAX_RANK, MAX_KEY, MAX_HEAD, MAX_VOCAB = 256, 512, 64, 128, 1 << 20

# The argument structs in the C compiler's layout (native alignment).  Packing
# 20 fields takes a fifth of the time of filling a ctypes structure, and small
# calls are bound by the host.
ROTARY = Struct("@PPPPqqqqqiiiiiiiif0q")
APPEND = Struct("@PPPPPPqqqqqqiiiiiif0q")
DECODE = Struct("@PPPPPPPNqqqqqqqqqqiiiiiiiif0q")
PREFILL = Struct("@PPPPPPPPqqqqqqqqqqqiiiiiiiif0q")
SAMPLE = Struct("@PPPPPPPPqiii0q")

EXPORTS = ["sim_op_rotary", "sim_op_latent_append", "sim_op_latent_decode", "sim_op_latent_decode_workspace",
           "sim_op_latent_prefill", "sim_op_sample", "sim_op_faults", "sim_op_last_error"]

_LIB = None
_WORKSPACE: dict[tuple, int] = {}  # bytes by sizes
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda device: torch.cuda.current_stream(device).cuda_stream)
# Scratch memory of the current device on a stream, without a tensor around it: 5 us less of a small call's 16.
_scratch = getattr(torch._C, "_cuda_cudaCachingAllocator_raw_alloc", None) or (
    lambda nbytes, stream: torch.cuda.caching_allocator_alloc(nbytes, stream=stream))
_changed = getattr(torch._C, "_increment_version", None) or torch.autograd.graph.increment_version  # of a tuple of tensors
_release = getattr(torch._C, "_cuda_cudaCachingAllocator_raw_delete", None) or torch.cuda.caching_allocator_delete


def lib() -> ctypes.CDLL:
    """libmtsim.so with the operators' entry points declared."""
    global _LIB
    if _LIB is None:
        L = mtsim.lib()
        for name in ("rotary", "latent_append", "latent_decode", "latent_prefill", "sample"):
            f = getattr(L, "sim_op_" + name)
            f.argtypes, f.restype = [ctypes.c_char_p, ctypes.c_void_p], ctypes.c_int
        L.sim_op_latent_decode_workspace.argtypes = [ctypes.c_int32] * 4
        L.sim_op_latent_decode_workspace.restype = ctypes.c_size_t
        L.sim_op_faults.argtypes, L.sim_op_faults.restype = [], ctypes.c_int
        L.sim_op_last_error.argtypes, L.sim_op_last_error.restype = [], ctypes.c_char_p
        _LIB = L
    return _LIB


def _failed(code: int):
    raise mtsim.SimError(code, lib().sim_op_last_error().decode())


def faults() -> int:
    """Waits inside the operators' kernels that ran out (0 unless a kernel is at fault); synchronises the device."""
    n = lib().sim_op_faults()
    if n < 0:
        _failed(n)
    return n


def _place(*tensors) -> int:
    """The one CUDA device, the current one, that every tensor is on; none may ask for a gradient."""
    device = tensors[0].get_device()
    for t in tensors:
        if t.get_device() != device:
            raise ValueError("every tensor must be on the same CUDA device")
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError("forward only: call under torch.no_grad() or detach the tensors")
    if forward_ad._current_level >= 0 and torch._C._is_fwd_grad_enabled():
        for t in tensors:
            if forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError("no forward-mode gradients: a tensor has a tangent")
    if device < 0:
        raise ValueError("the tensors must be on a CUDA device")
    if device != _current_device():
        raise ValueError("the tensors are on cuda:%d, which is not the current device" % device)
    return device


def _type(name, t, *others, wide=True) -> int:
    code = TYPES.get(t.dtype)
    if code is None or (code == 2 and not wide):
        raise TypeError("%s must be bfloat16 or float16%s, not %s" % (name, " or float32" if wide else "", t.dtype))
    for o in others:
        if o.dtype is not t.dtype:
            raise TypeError("tensors of one call must have the same type: %s and %s" % (t.dtype, o.dtype))
    return code


def _packed(name, t, shape) -> None:
    if t.shape != shape or not t.is_contiguous():
        raise ValueError("%s must be contiguous with shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))


def _rows(name, t, shape):
    """The strides of a tensor of that shape whose last dimension is contiguous."""
    s = t.stride()
    if t.shape != shape:
        raise ValueError("%s must have shape %s, not %s" % (name, tuple(shape), tuple(t.shape)))
    if s[-1] != 1 and shape[-1] > 1:
        raise ValueError("the last dimension of %s must be contiguous" % name)
    return s


def _positions(t, n) -> int:
    kind = t.dtype
    if kind is not torch.int32 and kind is not torch.int64:
        raise TypeError("positions must be int32 or int64, not %s" % kind)
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError("positions must be a contiguous vector of %d values" % n)
    return 1 if kind is torch.int64 else 0


def _frequencies(t) -> int:
    if t.dtype is not torch.float64 or t.dim() != 1 or not t.is_contiguous():
        raise ValueError("frequencies must be a contiguous float64 vector (see rotary_frequencies)")
    rot = 2 * t.shape[0]
    if not 2 <= rot <= MAX_ROT:
        raise ValueError("a rotated part has 2 to %d elements, not %d" % (MAX_ROT, rot))
    return rot


def _layout(name) -> int:
    code = LAYOUTS.get(name)
    if code is None:
        raise ValueError("layout must be 'interleaved' or 'half', not %r" % (name,))
    return code


def rotary_frequencies(rot_dim: int, base: float = 10000.0, *, scaling: str | None = None, factor: float = 1.0,
                       trained: int | None = None, fast: float = 32.0, slow: float = 1.0, device="cuda") -> torch.Tensor:
    """Radians per position of each pair of a rotated part, base^(-2i/rot_dim), in 64 bits.

    ``scaling`` stretches them for contexts ``factor`` times longer:
    ``"linear"`` divides all of them by ``factor``; ``"base"`` raises the base
    so that the slowest pair is slowed by ``factor`` and the fastest by nothing;
    ``"ramp"`` keeps the pairs that turn more than ``fast`` times over the
    ``trained`` length, divides those that turn less than ``slow`` times by
    ``factor``, and goes linearly in the number of turns from one to the other in
    between (use it with ``amplitude=ramp_amplitude(factor)``).  A model whose ramp
    was linear in the pair's index, or had its ends rounded to whole pairs, needs
    the vector that it was trained with: any float64 vector of radians per position does."""
    if rot_dim < 2 or rot_dim % 2 or rot_dim > MAX_ROT:
        raise ValueError("rot_dim must be even and in [2, %d]" % MAX_ROT)
    if not base > 0 or not factor > 0:
        raise ValueError("base and factor must be above zero")
    if scaling == "base" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = base ** (-torch.arange(rot_dim // 2, dtype=torch.float64) * 2 / rot_dim)
    if scaling == "linear":
        f = f / factor
    elif scaling == "ramp":
        if not trained or trained < 1 or not fast > slow:
            raise ValueError("the ramp needs the trained length, and fast > slow")
        slowed = ((fast - trained * f / (2 * math.pi)) / (fast - slow)).clamp(0, 1)
        f = f * (1 + (1 / factor - 1) * slowed)
    elif scaling not in (None, "base"):
        raise ValueError("scaling must be None, 'linear', 'base' or 'ramp', not %r" % (scaling,))
    return f.to(device)


def ramp_amplitude(factor: float) -> float:
    """The amplitude that goes with ``scaling="ramp"``: 0.1 ln(factor) + 1."""
    return 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0


def rotary(x, positions, frequencies, *, layout="interleaved", offset=0, amplitude=1.0, inverse=False, out=None):
    """Rotary positions on elements [offset, offset + 2 * len(frequencies)) of
    every head of ``x`` [tokens, heads, dim].  ``out=x`` works in place; the
    default is a new tensor, the other elements copied."""
    rot = _frequencies(frequencies)
    shape = x.shape
    if len(shape) != 3:
        raise ValueError("x must be [tokens, heads, dim]")
    n, heads, dim = shape
    if offset < 0 or offset + rot > dim:
        raise ValueError("elements [%d, %d) do not lie in a head of %d" % (offset, offset + rot, dim))
    wide = _positions(positions, n)
    if out is None:
        out = torch.empty(shape, dtype=x.dtype, device=x.device)
    xs, ys = _rows("x", x, shape), _rows("out", out, shape)
    code = _type("x", x, out)
    device = _place(x, out, positions, frequencies)
    rc = (_LIB or lib()).sim_op_rotary(
        ROTARY.pack(x.data_ptr(), out.data_ptr(), positions.data_ptr(), frequencies.data_ptr(), n, xs[0], xs[1], ys[0], ys[1],
                    heads, dim, rot, offset, code, _layout(layout), wide, 1 if inverse else 0, amplitude),
        _stream_of(device))
    if rc:
        _failed(rc)
    _changed((out,))
    return out


def latent_append(latent, key, positions, frequencies, slots, cache, *, layout="interleaved", amplitude=1.0):
    """Writes [latent[n], rotated key[n]] into row ``slots[n]`` (block *
    block_tokens + row) of ``cache`` [blocks, block_tokens, rank + rot]; a
    slot outside the cache (-1: padding) writes nothing.  Returns ``cache``."""
    rot = _frequencies(frequencies)
    if latent.dim() != 2 or cache.dim() != 3:
        raise ValueError("latent must be [tokens, rank], cache [blocks, block_tokens, rank + rot]")
    n, rank = latent.shape
    blocks, block, _ = cache.shape
    ls, ks = _rows("latent", latent, latent.shape), _rows("key", key, (n, rot))
    cs = _rows("cache", cache, (blocks, block, rank + rot))
    wide = _positions(positions, n)
    if slots.dtype is not torch.int64:
        raise TypeError("slots must be int64, not %s" % slots.dtype)
    _packed("slots", slots, (n,))
    code = _type("latent", latent, key, cache)
    device = _place(latent, key, cache, positions, frequencies, slots)
    rc = (_LIB or lib()).sim_op_latent_append(
        APPEND.pack(latent.data_ptr(), key.data_ptr(), cache.data_ptr(), positions.data_ptr(), slots.data_ptr(),
                    frequencies.data_ptr(), n, ls[0], ks[0], cs[0], cs[1], blocks, block, rank, rot, code, _layout(layout), wide,
                    amplitude),
        _stream_of(device))
    if rc:
        _failed(rc)
    _changed((cache,))
    return cache


def latent_decode(q, cache, table, lengths, *, scale, out=None, lse=None):
    """Attention of each request's newest tokens over its cached ones, in the
    absorbed form: ``q`` [requests, new, heads, width] are queries in the
    latent space, ``cache`` [blocks, block_tokens, width] holds a latent
    vector and the rotated shared key a row, ``table`` int32 [requests, n]
    names each request's blocks, ``lengths`` int32 [requests] counts cached
    tokens, the new ones included.  The values are the rows' first ``rank``
    elements, ``rank`` being ``out``'s last dimension (default: width - 64).
    Returns (out [requests, new, heads, rank], lse float32)."""
    if q.dim() != 4 or cache.dim() != 3 or table.dim() != 2:
        raise ValueError("q must be [requests, new, heads, width], cache [blocks, block_tokens, width], table [requests, n]")
    b, new, heads, width = q.shape
    blocks, block, _ = cache.shape
    if out is None:
        out = torch.empty((b, new, heads, width - 64), dtype=q.dtype, device=q.device)
    rank = out.shape[-1]
    if rank < 64 or rank > MAX_RANK or rank % 64 or not 0 <= width - rank <= MAX_KEY or width % 8:
        raise ValueError("rank must be a multiple of 64 up to %d and width - rank one of 8 up to %d: %d, %d"
                         % (MAX_RANK, MAX_KEY, rank, width - rank))
    qs, os_ = _rows("q", q, q.shape), _rows("out", out, (b, new, heads, rank))
    cs = _rows("cache", cache, (blocks, block, width))
    ts = _rows("table", table, (b, table.shape[1]))
    if table.dtype is not torch.int32 or lengths.dtype is not torch.int32:
        raise TypeError("table and lengths must be int32")
    _packed("lengths", lengths, (b,))
    if lse is None:
        lse = torch.empty((b, new, heads), dtype=torch.float32, device=q.device)
    elif lse.dtype is not torch.float32:
        raise TypeError("lse must be float32")
    _packed("lse", lse, (b, new, heads))
    code = _type("q", q, cache, out, wide=False)
    device = _place(q, cache, out, lse, table, lengths)
    L = _LIB or lib()
    size = (device, b, new, heads, rank)
    nbytes = _WORKSPACE.get(size)
    if nbytes is None:
        nbytes = L.sim_op_latent_decode_workspace(b, new, heads, rank)
        if not nbytes:  # the device could not be asked: not an answer to keep
            _failed(mtsim.SIM_ERR_CUDA)
        _WORKSPACE[size] = nbytes
    stream = _stream_of(device)
    work = _scratch(nbytes, stream)
    try:
        rc = L.sim_op_latent_decode(
            DECODE.pack(q.data_ptr(), cache.data_ptr(), table.data_ptr(), lengths.data_ptr(), out.data_ptr(), lse.data_ptr(),
                        work, nbytes, qs[0], qs[1], qs[2], os_[0], os_[1], os_[2], cs[0], cs[1], ts[0], blocks, b, new,
                        heads, rank, width - rank, block, table.shape[1], code, scale),
            stream)
    finally:
        _release(work)  # what the stream allocates next comes after this call's kernels
    if rc:
        _failed(rc)
    _changed((out, lse))
    return out, lse


def latent_prefill(q, key, shared, value, q_offsets, k_offsets, *, scale, longest, causal=True, out=None, lse=None):
    """Attention of ragged prompts with expanded keys and values: ``q`` [rows,
    heads, head_dim + key_dim], ``key`` [k_rows, heads, head_dim], ``shared``
    [k_rows, key_dim] (the rotated key of every head), ``value`` [k_rows,
    heads, value_dim].  Request b has the rows between ``q_offsets[b]`` and
    ``[b + 1]`` (int32) and likewise keys; the last query sees every key
    and each earlier one a key less (``causal=False``: all of them).
    ``longest`` bounds a request's queries.  Returns (out [rows, heads,
    value_dim], lse float32 [rows, heads])."""
    if q.dim() != 3 or key.dim() != 3 or shared.dim() != 2 or value.dim() != 3:
        raise ValueError("q, key and value must be [rows, heads, dim], shared [rows, dim]")
    n, heads, width = q.shape
    m, _, head = key.shape
    rot, wide = shared.shape[1], value.shape[2]
    if width != head + rot:
        raise ValueError("q's heads have %d elements, key and shared %d + %d" % (width, head, rot))
    if out is None:
        out = torch.empty((n, heads, wide), dtype=q.dtype, device=q.device)
    qs, ks = _rows("q", q, q.shape), _rows("key", key, (m, heads, head))
    ss, vs = _rows("shared", shared, (m, rot)), _rows("value", value, (m, heads, wide))
    os_ = _rows("out", out, (n, heads, wide))
    if q_offsets.dtype is not torch.int32 or k_offsets.dtype is not torch.int32:
        raise TypeError("q_offsets and k_offsets must be int32")
    b = q_offsets.shape[0] - 1
    if b < 0:
        raise ValueError("offsets have one entry more than there are requests")
    _packed("q_offsets", q_offsets, (b + 1,))
    _packed("k_offsets", k_offsets, (b + 1,))
    if lse is None:
        lse = torch.empty((n, heads), dtype=torch.float32, device=q.device)
    elif lse.dtype is not torch.float32:
        raise TypeError("lse must be float32")
    _packed("lse", lse, (n, heads))
    code = _type("q", q, key, shared, value, out, wide=False)
    device = _place(q, key, shared, value, out, lse, q_offsets, k_offsets)
    rc = (_LIB or lib()).sim_op_latent_prefill(
        PREFILL.pack(q.data_ptr(), key.data_ptr(), shared.data_ptr(), value.data_ptr(), q_offsets.data_ptr(),
                     k_offsets.data_ptr(), out.data_ptr(), lse.data_ptr(), qs[0], qs[1], ks[0], ks[1], ss[0], vs[0], vs[1],
                     os_[0], os_[1], n, m, b, heads, longest, head, rot, wide, 1 if causal else 0, code, scale),
        _stream_of(device))
    if rc:
        _failed(rc)
    _changed((out, lse))
    return out, lse


def sample(logits, uniform, *, temperature=None, top_k=None, top_p=None, min_p=None, out=None, logprob=None):
    """One token per row of ``logits`` [rows, vocab] from the given ``uniform``
    float32 [rows] in [0, 1).  ``temperature``, ``top_p``, ``min_p`` (float32)
    and ``top_k`` (int32) are vectors of one value a row, or None; a
    temperature of zero takes the largest logit.  The draw goes through the kept tokens in
    vocabulary order.  Returns (token int64 [rows], logprob float32 [rows]);
    a row without a finite logit gives -1."""
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, vocab]")
    rows, vocab = logits.shape
    if not 1 <= vocab <= MAX_VOCAB:
        raise ValueError("a vocabulary has 1 to %d tokens, not %d" % (MAX_VOCAB, vocab))
    stride = _rows("logits", logits, logits.shape)[0]
    if out is None:
        out = torch.empty(rows, dtype=torch.int64, device=logits.device)
    if logprob is None:
        logprob = torch.empty(rows, dtype=torch.float32, device=logits.device)
    code = _type("logits", logits)
    used = [logits]

    def vector(name, t, dtype):
        """The address of a vector of one value a row (0: none)."""
        if t is None:
            return 0
        if t.dtype is not dtype:
            raise TypeError("%s must be %s, not %s" % (name, dtype, t.dtype))
        if t.dim() != 1 or t.shape[0] != rows or not t.is_contiguous():
            raise ValueError("%s must be a contiguous vector of %d values" % (name, rows))
        used.append(t)
        return t.data_ptr()

    real = torch.float32
    args = SAMPLE.pack(logits.data_ptr(), vector("uniform", uniform, real), vector("temperature", temperature, real),
                       vector("top_k", top_k, torch.int32), vector("top_p", top_p, real), vector("min_p", min_p, real),
                       vector("out", out, torch.int64), vector("logprob", logprob, real), stride, rows, vocab, code)
    device = _place(*used)
    rc = (_LIB or lib()).sim_op_sample(args, _stream_of(device))
    if rc:
        _failed(rc)
    _changed((out, logprob))
    return out, logprob
