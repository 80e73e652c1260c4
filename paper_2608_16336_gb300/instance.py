"""One serving instance run for real, to time the iterations that the simulator charges.

The simulator's instances form a batch, prefill the admitted prompts, advance
every running request by a token and are busy for base + a * prefill tokens +
b * decode requests microseconds (Sec. 2.2, 3.1).  The paper's simulator takes
such times from operators profiled on a GPU (Sec. 2.5, 4.1).  ``Instance``
executes that iteration with the operators of ``instance_ops`` over a block
cache of the simulated shape (M blocks of T tokens, Bmax requests), ``measure``
times iterations of mixed batches, ``fit_iteration_times`` gives base, a and b, and
``with_times`` puts them into a workload::

    from paper_2608_16336_gb300 import instance, mtsim, workloads

    w = workloads.config(1, replicas=range(8), requests=500)
    node = instance.Instance(instance.Shape(layers=24), blocks=w.blocks_per_instance,
                             block_tokens=w.tokens_per_block, max_batch=w.max_batch)
    times = instance.fit_iteration_times(instance.measure(node), per_us=10)
    sim = mtsim.Simulator(instance.with_times(w, times, per_us=10))  # in tenths of a microsecond

Weights are random; the layers are attention layers with their projections
(plain matrix products), and ``feed_forward`` adds what else a layer does.

An instance's cache is of the shape's type, or (``quantized``) of 8-bit
numbers with scales.  ``speculate`` advances the running requests by drafted
tokens, ``fork`` lets requests share their blocks, ``migrate`` moves one to
another instance's cache and ``compact`` the used blocks to the start.
"""
from __future__ import annotations

import dataclasses
import itertools
import math
import warnings

import numpy as np
import torch

from . import instance_ops as ops


@dataclasses.dataclass(frozen=True)
class Shape:
    """A model's attention: every cached token is ``rank`` + ``key_dim`` elements, shared by the heads."""

    layers: int = 2
    hidden: int = 2048
    heads: int = 16
    head_dim: int = 128
    key_dim: int = 64
    value_dim: int = 128
    rank: int = 512
    vocab: int = 32000
    base: float = 10000.0
    layout: str = "half"
    dtype: torch.dtype = torch.bfloat16


@dataclasses.dataclass
class Running:
    """A request in the cache: its blocks, tokens held, and the last token drawn."""

    blocks: list[int]
    length: int
    token: torch.Tensor


def _norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Instance:
    """An instance with ``blocks`` cache blocks of ``block_tokens`` tokens and at
    most ``max_batch`` running requests, on the current CUDA device;
    ``quantized`` holds the cache in 8 bits (``instance_ops.quantized_append``)."""

    shared: dict[int, int] = {}  # blocks that more than one request holds, by how many more; replaced, never changed in place
    scales = None

    def __init__(self, shape: Shape = Shape(), *, blocks: int, block_tokens: int, max_batch: int = 64, seed: int = 0,
                 frequencies: torch.Tensor | None = None, feed_forward=None, quantized: bool = False):
        if blocks < 1 or block_tokens < 1 or max_batch < 1:
            raise ValueError("blocks, block_tokens and max_batch must be at least 1")
        self.shape, self.block_tokens, self.max_batch, self.feed_forward = shape, block_tokens, max_batch, feed_forward
        self.free = list(range(blocks))[::-1]
        self.running: dict[int, Running] = {}
        self._next = 0
        self.frequencies = ops.rotary_frequencies(shape.key_dim, shape.base) if frequencies is None else frequencies
        self.scale = 1.0 / math.sqrt(shape.head_dim + shape.key_dim)
        s, g = shape, torch.Generator(device="cuda").manual_seed(seed)

        def weight(*size, fan):
            return (torch.randn(size, generator=g, device="cuda") / math.sqrt(fan)).to(s.dtype)

        self.embed = weight(s.vocab, s.hidden, fan=1)
        self.layers = [dict(q=weight(s.hidden, s.heads * (s.head_dim + s.key_dim), fan=s.hidden),
                            kv=weight(s.hidden, s.rank + s.key_dim, fan=s.hidden),
                            key_up=weight(s.heads, s.rank, s.head_dim, fan=s.rank),
                            value_up=weight(s.heads, s.rank, s.value_dim, fan=s.rank),
                            out=weight(s.heads * s.value_dim, s.hidden, fan=s.heads * s.value_dim)) for _ in range(s.layers)]
        size = s.layers, blocks, block_tokens, s.rank + s.key_dim
        if quantized:  # (bytes of 0 are zeros)
            self.cache = torch.zeros(size, dtype=torch.uint8, device="cuda").view(ops.EIGHT)
            self.scales = torch.ones(s.layers, blocks, 2, device="cuda")
        else:
            self.cache = torch.zeros(size, dtype=s.dtype, device="cuda")
        self.unembed = weight(s.hidden, s.vocab, fan=s.hidden)

    # -- the cache
    def blocks_for(self, tokens: int) -> int:
        return -(-tokens // self.block_tokens)

    def _plan(self, held, lengths):
        """Every request's blocks with room for ``lengths`` tokens, ``held``
        being those it has, and how many come from the end of the free list.
        Changes nothing: an iteration that does not fit is refused here."""
        need = [self.blocks_for(n) - len(b) for b, n in zip(held, lengths)]
        wanted, taken, blocks = sum(need), 0, []
        if wanted > len(self.free):
            raise RuntimeError("out of cache blocks: %d wanted, %d free" % (wanted, len(self.free)))
        for b, k in zip(held, need):
            blocks.append(b + [self.free[-1 - i] for i in range(taken, taken + k)])
            taken += k
        return blocks, taken

    def _give_back(self, blocks) -> None:
        """Frees blocks, those alone that no other request holds."""
        shared = dict(self.shared)
        for b in blocks:
            if b not in shared:
                self.free.append(b)
            elif shared[b] > 1:
                shared[b] -= 1
            else:
                del shared[b]
        self.shared = shared

    def _own(self, blocks, first, taken):
        """``blocks`` with those that a request is about to write (from its
        token ``first`` on) and others hold too replaced by free ones, how many free
        ones are taken with these, and the pairs to be copied.  Changes nothing."""
        if not self.shared:
            return blocks, taken, []
        copies, blocks = [], [list(b) for b in blocks]
        left = dict(self.shared)
        for b, n in zip(blocks, first):
            for i in range(n // self.block_tokens, len(b)):
                if left.get(b[i]):
                    if taken >= len(self.free):
                        raise RuntimeError("out of cache blocks: none is free for a block that requests share")
                    left[b[i]] -= 1
                    copies.append((b[i], self.free[-1 - taken]))
                    b[i] = self.free[-1 - taken]
                    taken += 1
        return blocks, taken, copies

    def _copy(self, pairs, other=None) -> None:
        """Copies blocks of the cache, and their scales, to blocks of ``other``'s (default: this one's)."""
        if pairs:
            other = self if other is None else other
            a, b = torch.tensor(list(zip(*pairs)), dtype=torch.int32, device="cuda")
            ops.block_copy(self.cache, other.cache, a, b)
            if self.scales is not None:
                ops.block_copy(self.scales, other.scales, a, b)

    def release(self, request: int) -> None:
        """Takes a request out of the batch and gives its blocks back."""
        self._give_back(self.running.pop(request).blocks[::-1])

    def rewind(self, request: int, tokens: int) -> None:
        """Takes a running request back to its first ``tokens`` cached tokens."""
        q = self.running[request]
        if not 1 <= tokens <= q.length:
            raise ValueError("a request of %d tokens cannot go back to %d" % (q.length, tokens))
        q.length = tokens
        keep = self.blocks_for(tokens)
        self._give_back(q.blocks[keep:][::-1])
        del q.blocks[keep:]

    def fork(self, request: int, copies: int = 1) -> list[int]:
        """Adds ``copies`` requests that go on from where ``request`` is, with its
        full blocks; a block that is not full is copied.  Returns their numbers."""
        q = self.running[request]
        if copies < 1 or len(self.running) + copies > self.max_batch:
            raise ValueError("more than max_batch = %d requests, or no copy" % self.max_batch)
        part = q.length % self.block_tokens > 0
        if part and copies > len(self.free):
            raise RuntimeError("out of cache blocks: %d wanted, %d free" % (copies, len(self.free)))
        own = [self.free[-1 - i] for i in range(copies)] if part else [None] * copies
        self._copy([(q.blocks[-1], b) for b in own] if part else [])
        if part:
            del self.free[len(self.free) - copies:]
        full, ids = q.blocks[:-1] if part else q.blocks, []
        self.shared = {**self.shared, **{b: self.shared.get(b, 0) + copies for b in full}}
        for b in own:
            self.running[self._next] = Running(full + ([b] if part else []), q.length, q.token)
            ids.append(self._next)
            self._next += 1
        return ids

    def migrate(self, request: int, other: "Instance") -> int:
        """Moves a running request into ``other``'s batch and cache; returns its number there."""
        if other is self or self.shape != other.shape or self.block_tokens != other.block_tokens or (self.scales is None) != (other.scales is None):
            raise ValueError("a request moves to another instance with the same shape, block size and cache type")
        if len(other.running) >= other.max_batch:
            raise ValueError("more than max_batch = %d requests" % other.max_batch)
        q = self.running[request]
        (blocks,), taken = other._plan([[]], [q.length])
        self._copy(list(zip(q.blocks, blocks)), other)
        del other.free[len(other.free) - taken:]
        there, other._next = other._next, other._next + 1
        other.running[there] = Running(blocks, q.length, q.token)
        self.release(request)
        return there

    def compact(self) -> int:
        """Moves the used blocks to the start of the cache; returns how many moved."""
        used = sorted({b for q in self.running.values() for b in q.blocks})
        holes = sorted(set(range(len(used))) - set(used))
        to = dict(zip([b for b in used if b >= len(used)], holes))
        self._copy(list(to.items()))
        for q in self.running.values():
            q.blocks = [to.get(b, b) for b in q.blocks]
        self.shared = {to.get(b, b): n for b, n in self.shared.items()}
        self.free = list(range(len(used), len(used) + len(self.free)))[::-1]
        return len(to)

    # -- an iteration
    @torch.no_grad()
    def iterate(self, prompts=(), *, uniform: torch.Tensor | None = None, temperature=None, top_k=None, top_p=None, min_p=None,
                advance: bool = True):
        """One iteration: prefills ``prompts`` (int64 token vectors on the device),
        advances every running request by its last token (``advance=False``:
        none), and draws the next token of all of them.  Returns (requests, tokens, log-probabilities),
        the running ones first; the prompts are running from then on.
        ``uniform`` gives the draws (default: from PyTorch's generator), the
        others are vectors as in ``instance_ops.sample``, one value a request.
        A call that raises leaves the batch and the free blocks as they were."""
        prompts = list(prompts)
        if any(len(p) < 1 for p in prompts):
            raise ValueError("a prompt has at least one token")
        if len(self.running) + len(prompts) > self.max_batch:
            raise ValueError("more than max_batch = %d requests" % self.max_batch)
        decode = list(self.running) if advance else []
        if not decode and not prompts:
            raise ValueError("nothing to do: no prompt and no running request")
        lengths = [self.running[r].length + 1 for r in decode] + [len(p) for p in prompts]
        blocks, taken = self._plan([self.running[r].blocks for r in decode] + [[] for _ in prompts], lengths)
        blocks, taken, copies = self._own(blocks, [self.running[r].length for r in decode] + [0] * len(prompts), taken)

        nd = len(decode)
        where = self._where(blocks, lengths, nd, 1, prompts)
        last = list(range(nd)) + (np.cumsum([len(p) for p in prompts], dtype=np.int64) + (nd - 1)).tolist()
        last = torch.tensor(last, dtype=torch.int64, device="cuda")
        self._copy(copies)
        x = self.embed[torch.cat([self.running[r].token for r in decode] + prompts)]
        x = self._forward(x, where, nd, 1, prompts)
        logits = _norm(x[last]) @ self.unembed
        if uniform is None:
            uniform = torch.rand(len(logits), device="cuda")
        tokens, logprob = ops.sample(logits, uniform, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
        # everything is queued: the batch changes now
        del self.free[len(self.free) - taken:]
        self._give_back([b for b, _ in copies])
        ids = decode + list(range(self._next, self._next + len(prompts)))
        self._next += len(prompts)
        for i, (r, b, n) in enumerate(zip(ids, blocks, lengths)):
            self.running[r] = Running(b, n, tokens[i:i + 1])
        return ids, tokens, logprob

    @torch.no_grad()
    def speculate(self, drafts: torch.Tensor, *, draft: torch.Tensor | None = None, uniform: torch.Tensor | None = None, temperature=None):
        """One iteration in which every running request advances by its last
        token and as many of its drafted ones (int64 [requests, n]; they end at the first -1 or other number outside the vocabulary) as
        ``instance_ops.verify`` accepts, with the token that follows them.  ``draft``, ``uniform`` and
        ``temperature`` as there (default: certain drafts, draws from PyTorch's generator).  Tokens follow the target's whole
        distribution: there is no top-k, top-p or min-p as in ``iterate``.  Returns (requests,
        tokens [requests, n + 1], -1 behind each request's; how many, on the host; log-probabilities).
        A call that raises leaves the batch and the free blocks as they were."""
        ids = list(self.running)
        if drafts.dim() != 2 or drafts.shape[0] != len(ids) or not ids:
            raise ValueError("drafts must be [running requests, n], and a request must be running")
        new = drafts.shape[1] + 1
        held = [self.running[r].length for r in ids]
        lengths = [n + new for n in held]
        blocks, taken = self._plan([self.running[r].blocks for r in ids], lengths)
        blocks, taken, copies = self._own(blocks, held, taken)
        where = self._where(blocks, lengths, len(ids), new, [])
        self._copy(copies)
        x = self.embed[torch.cat((torch.stack([self.running[r].token for r in ids]), drafts.clamp(0, len(self.embed) - 1)), 1).flatten()]
        x = self._forward(x, where, len(ids), new, [])
        target = (_norm(x) @ self.unembed).view(len(ids), new, -1)
        if uniform is None:
            uniform = torch.rand(len(ids), new, device="cuda")
        # a request's drafts end at the first that is none: the token in its place is the target's, whatever the draft's row holds
        drafted = ((drafts >= 0) & (drafts < target.shape[-1])).cumprod(1).sum(1, dtype=torch.int32)
        tokens, count, logprob = ops.verify(target, drafts.contiguous(), uniform, draft=draft, temperature=temperature, drafted=drafted)
        counts = count.tolist()
        del self.free[len(self.free) - taken:]
        self._give_back([b for b, _ in copies])
        for i, (r, b, n) in enumerate(zip(ids, blocks, held)):
            self.running[r] = Running(b, lengths[i], tokens[i, counts[i] - 1:counts[i]])
            self.rewind(r, n + counts[i])
        return ids, tokens, counts, logprob

    def _where(self, blocks, lengths, nd, new, prompts):
        """What the kernels read of ``nd`` requests' last ``new`` tokens each, then
        the prompts, ``lengths`` counting every request's tokens with them: positions, slots, lengths, the running requests' table (and the
        prompts', to an 8-bit cache), every request's first row, the prompts' first rows and the longest.
        (A copy to the device waits for the stream: all of them come before the first kernel.)"""
        quantized = self.scales is not None
        put = lambda v, dtype: torch.tensor(v, dtype=dtype, device="cuda")
        positions, slots = _places(blocks, lengths, nd, new, self.block_tokens)
        named = blocks if quantized else blocks[:nd]
        widest = max((len(b) for b in named), default=0)
        table = put([b + [0] * (widest - len(b)) for b in named], torch.int32).reshape(len(named), widest)
        offsets = np.cumsum([0] + [len(p) for p in prompts])
        rows = [new * i for i in range(nd)] + (nd * new + offsets).tolist()
        return (put(positions, torch.int32), None if quantized else put(slots, torch.int64), put(lengths if quantized else lengths[:nd], torch.int32), table,
                put(rows, torch.int32) if quantized else None, put(offsets.tolist(), torch.int32), max((len(p) for p in prompts), default=0))

    def _forward(self, x, where, nd, new, prompts):
        """The layers over ``nd`` requests' last ``new`` tokens each, then the prompts."""
        s, n, rows, quantized = self.shape, x.shape[0], nd * new, self.scales is not None
        positions, slots, every, table, all_starts, starts, longest = where
        for i, (layer, cache) in enumerate(zip(self.layers, self.cache)):
            h = _norm(x)
            q = (h @ layer["q"]).view(n, s.heads, s.head_dim + s.key_dim)
            kv = h @ layer["kv"]
            latent, key = _norm(kv[:, :s.rank]), kv[:, s.rank:]
            ops.rotary(q, positions, self.frequencies, layout=s.layout, offset=s.head_dim, out=q)
            if quantized:
                ops.quantized_append(latent, key, self.frequencies, all_starts, table, every, cache, self.scales[i], layout=s.layout)
            else:
                ops.latent_append(latent, key, positions, self.frequencies, slots, cache, layout=s.layout)
            out = torch.empty(n, s.heads, s.value_dim, dtype=s.dtype, device="cuda")
            if nd:  # absorbed: queries go into the latent space, values come out of it
                inner = torch.matmul(q[:rows, :, :s.head_dim].transpose(0, 1), layer["key_up"].transpose(1, 2)).transpose(0, 1)
                inner = torch.cat((inner, q[:rows, :, s.head_dim:]), -1).unflatten(0, (nd, new))
                got = torch.empty(nd, new, s.heads, s.rank, dtype=s.dtype, device="cuda")
                if quantized:
                    ops.quantized_decode(inner, cache, self.scales[i], table[:nd], every[:nd], scale=self.scale, out=got)
                else:
                    ops.latent_decode(inner, cache, table, every, scale=self.scale, out=got)
                out[:rows] = torch.matmul(got.flatten(0, 1).transpose(0, 1), layer["value_up"]).transpose(0, 1)
            if prompts:  # expanded: every head has keys and values of its own
                keys = torch.matmul(latent[rows:], layer["key_up"]).transpose(0, 1)
                values = torch.matmul(latent[rows:], layer["value_up"]).transpose(0, 1)
                shared = ops.rotary(key[rows:, None], positions[rows:], self.frequencies, layout=s.layout)[:, 0]
                ops.latent_prefill(q[rows:], keys, shared, values, starts, starts, scale=self.scale, longest=longest, out=out[rows:])
            x = x + out.flatten(1) @ layer["out"]
            if self.feed_forward is not None:
                x = self.feed_forward(x)
        return x


def _places(blocks, lengths, nd, new, t):
    """Positions and slots of ``nd`` requests' last ``new`` tokens each, then of whole prompts, in blocks of ``t`` tokens."""
    positions, slots = [], []
    for b, k in zip(blocks[:nd], lengths):  # (a long request's blocks are not gone through for a token)
        for p in range(k - new, k):
            positions.append(p)
            slots.append(b[p // t] * t + p % t)
    for b, k in zip(blocks[nd:], lengths[nd:]):
        at = np.arange(k)
        positions += at.tolist()
        slots += (np.asarray(b)[at // t] * t + at % t).tolist()
    return positions, slots


def measure(node: Instance, *, prefill_tokens=(0, 256, 1024, 4096), decodes=(0, 8, 32, 63), context: int = 512, repeats: int = 3):
    """Times iterations of ``node``: for every pair of prefill tokens (one
    prompt) and decode requests (each with ``context`` cached tokens before the
    iteration), the median of ``repeats`` iterations in microseconds, from CUDA events, host
    work included.  Returns [(prefill tokens, decode requests, microseconds)];
    pairs that do not fit the instance are left out.  The instance has no
    running requests afterwards, also where an iteration raises."""
    if node.running:
        raise ValueError("the instance has running requests")
    if context < 1 or repeats < 1:
        raise ValueError("context and repeats must be at least 1")
    g = torch.Generator(device="cuda").manual_seed(1)
    prompt = lambda n: torch.randint(0, node.shape.vocab, (n,), generator=g, device="cuda")
    fits = lambda p, d: d + (p > 0) <= node.max_batch and d * node.blocks_for(context + 1) + node.blocks_for(p) <= blocks
    blocks, samples, faults = len(node.free), [], ops.faults()
    try:
        for d in decodes:
            if not any(fits(p, d) for p in prefill_tokens if p or d):
                continue
            for _ in range(d):  # one at a time: a prefill of all would need them expanded at once
                node.iterate([prompt(context)], advance=False)
            held = list(node.running)
            for p in prefill_tokens:
                if not (p or d) or not fits(p, d):
                    continue
                times = []
                for _ in range(repeats + 1):  # the first warms up
                    new = [prompt(p)] if p else []
                    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
                    torch.cuda.synchronize()
                    a.record()
                    ids, _, _ = node.iterate(new)
                    b.record()
                    b.synchronize()
                    times.append(a.elapsed_time(b) * 1e3)
                    for r in held:
                        node.rewind(r, context)
                    if p:
                        node.release(ids[-1])
                samples.append((p, d, float(np.median(times[1:]))))
            for r in held:
                node.release(r)
    finally:
        for r in list(node.running):
            node.release(r)
    if ops.faults() != faults:
        raise RuntimeError("a wait inside a kernel ran out: the times are not to be used")
    return samples


def fit_iteration_times(samples, *, per_us: int = 1):
    """The integer constants (base, a, b) of base + a * prefill tokens + b *
    decode requests nearest to the samples (least squares of relative errors,
    none below zero), in units of 1 / ``per_us`` microseconds: the simulator's
    times are whole numbers, and a token often costs less than a microsecond.
    Warns where whole units move the time of a sample by more than 5 %;
    ``with_times`` takes the same ``per_us``."""
    if per_us < 1 or int(per_us) != per_us:
        raise ValueError("per_us must be a whole number of units, at least 1")
    m = np.array([[1.0, p, d] for p, d, _ in samples])
    t = np.array([x for _, _, x in samples], dtype=np.float64) * per_us
    if len(t) < 3 or not (t > 0).all():
        raise ValueError("three samples or more with times above zero are needed")

    rows, best, real = m / t[:, None], math.inf, None
    off = lambda x: float(((rows @ x - 1) ** 2).sum())
    for keep in itertools.chain.from_iterable(itertools.combinations(range(3), k) for k in (3, 2, 1)):
        x = np.zeros(3)
        x[list(keep)] = np.linalg.lstsq(rows[:, keep], np.ones_like(t), rcond=None)[0]
        if (x >= 0).all() and off(x) < best - 1e-12:
            best, real = off(x), x
    # whole numbers: the pairs (a, b) around, each with its own best base
    best, found = math.inf, None
    around = lambda v: range(max(0, math.floor(v) - 3), math.floor(v) + 5)
    for a, b in itertools.product(around(real[1]), around(real[2])):
        rest = 1 - rows[:, 1] * a - rows[:, 2] * b
        x = np.array([max(1.0, np.rint(rows[:, 0] @ rest / (rows[:, 0] @ rows[:, 0]))), a, b])
        if off(x) < best:
            best, found = off(x), x
    moved = float((np.abs(m @ found - m @ real) / t).max())
    if moved > 0.05:
        warnings.warn("whole %s move a sample's time by %.0f %%; a larger per_us holds what was measured"
                      % ("microseconds" if per_us == 1 else "units of 1/%d us" % per_us, 100 * moved), RuntimeWarning, stacklevel=2)
    return tuple(int(v) for v in found)


def with_times(w, times, *, per_us: int = 1):
    """A copy of workload ``w`` whose iterations take the given (base, a, b),
    constants in units of 1 / ``per_us`` microseconds as
    ``fit_iteration_times`` gives them.  All of the copy's times are in that
    unit then (arrivals, the migration interval and drain times are
    multiplied), and so are the times that its simulation reports."""
    times = dict(iter_base_us=int(times[0]), iter_us_per_prefill_token=int(times[1]), iter_us_per_decode_seq=int(times[2]))
    if per_us < 1 or int(per_us) != per_us:
        raise ValueError("per_us must be a whole number of units, at least 1")
    if per_us == 1:
        return dataclasses.replace(w, **times)
    never = 0xFFFFFFFF

    def scaled(v):
        v = np.asarray(v)
        x = np.where(v == never, never, v.astype(np.uint64) * np.uint64(per_us))
        if ((x >= never) & (v != never)).any():
            raise ValueError("times in units of 1/%d us pass 32 bits" % per_us)
        return x.astype(v.dtype)

    return dataclasses.replace(w, **times, migrate_interval_us=w.migrate_interval_us * per_us, arrival_us=scaled(w.arrival_us),
                               drain_start_us=None if w.drain_start_us is None else scaled(w.drain_start_us))
