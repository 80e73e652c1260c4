"""Performance cases of an instance's operators for 8-bit caches, drafted tokens and moved blocks.

The simulator's instances keep their requests' keys and values in blocks of T
tokens, run iterations of prefills and single tokens, and move blocks from one
instance to another.  These cases time on the device:

* ``append``: new tokens' latent vectors and rotated shared keys into a block
  cache of 8-bit numbers with a scale for each block and part (latent, key);
* ``decode``: attention of new tokens over such a cache, queries already in
  the latent space (the absorbed form);
* ``verify``: drafted tokens against the target's probabilities, from given
  uniform numbers, with the token that follows the accepted ones;
* ``copy``: blocks of all layers to other blocks of the same or another cache.

A case's lengths come from the case alone and its values from the seed.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}
LARGEST = 448.0  # of the 8-bit type


def _append(name, requests, shortest, longest, cached, rank, rot, block, layout, dtype):
    return dict(name=name, op="append", requests=requests, shortest=shortest, longest=longest, cached=cached, rank=rank, rot=rot,
                block=block, layout=layout, dtype=dtype)


def _decode(name, requests, new, heads, rank, rot, block, shortest, longest, empty, dtype):
    return dict(name=name, op="decode", requests=requests, new=new, heads=heads, rank=rank, rot=rot, block=block,
                shortest=shortest, longest=longest, empty=empty, dtype=dtype)


def _verify(name, requests, drafts, vocab, ragged, known, temperature, spread, dtype):
    return dict(name=name, op="verify", requests=requests, drafts=drafts, vocab=vocab, ragged=ragged, known=known,
                temperature=temperature, spread=spread, dtype=dtype)


def _copy(name, layers, blocks, pairs, block, width, inside, padding, dtype):
    return dict(name=name, op="copy", layers=layers, blocks=blocks, pairs=pairs, block=block, width=width, inside=inside,
                padding=padding, dtype=dtype)


def listed():
    return [
        # one iteration of a full running batch: a token each, most of them into blocks that hold rows already
        _append("append_batch", 64, 1, 1, 10240, 512, 64, 16, "interleaved", "bf16"),
        # prompts and chunks of prompts of one iteration, beginning and ending inside blocks of 12
        _append("append_prompts", 9, 300, 8191, 4100, 512, 64, 12, "half", "fp16"),
        # one lightly loaded request with a short context
        _decode("decode_one", 1, 1, 16, 512, 64, 16, 777, 777, 0, "bf16"),
        # a full running batch with every head on this GPU, prompts as in the long-prompt traces, some slots empty
        _decode("decode_batch", 64, 1, 128, 512, 64, 16, 200, 10240, 3, "bf16"),
        # part of a batch with four drafted tokens a request
        _decode("decode_drafts", 23, 5, 16, 512, 64, 16, 1000, 10240, 1, "bf16"),
        # a few requests with very long contexts and two new tokens each
        _decode("decode_long", 3, 2, 16, 512, 64, 64, 90001, 130000, 0, "fp16"),
        # one request's four drafted tokens
        _verify("verify_one", 1, 4, 32000, False, True, 0.8, 3.0, "fp32"),
        # the running batch, a large vocabulary
        _verify("verify_batch", 64, 3, 131075, False, True, 0.9, 2.0, "bf16"),
        # drafts looked up in the prompt, up to eight of them and no draft distribution, some requests greedy
        _verify("verify_lookup", 37, 8, 50001, True, False, 0.7, 4.0, "fp16"),
        # every request of a batch forked: its last block in every layer
        _copy("copy_fork", 8, 2048, 64, 16, 576, True, 0, "bf16"),
        # a long request migrated to another instance: all its blocks
        _copy("copy_migrate", 24, 2048, 640, 16, 576, False, 0, "bf16"),
        # a cache compacted: scattered blocks of 12 rows of 8-bit numbers, the list padded
        _copy("copy_compact", 27, 4096, 1500, 12, 560, True, 100, "e4m3"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi + 0.49))))))


def draw(rng):
    op, wide = rng.choice(("append", "decode", "verify", "copy")), rng.choice(("bf16", "fp16"))
    if op == "append":
        requests = _log_int(rng, 1, 200)
        longest = 1 if rng.random() < 0.4 else _log_int(rng, 2, max(2, min(16384, 30000 // requests)))
        c = _append("", requests, max(1, longest // rng.choice((1, 5, 40))), longest, _log_int(rng, 1, min(20000, 600000 // requests)),
                    rng.choice((128, 256, 512, 512)), rng.choice((32, 64, 64)), rng.choice((8, 12, 16, 16, 32, 64)),
                    rng.choice(("interleaved", "half")), rng.choice(("bf16", "fp16", "fp32")))
    elif op == "decode":
        requests, new, heads = _log_int(rng, 1, 64), rng.choice((1, 1, 1, 2, 3, 5)), _log_int(rng, 1, 128)
        most = max(64, min(130000, 64 * 10240 // (2 * requests), 64 * 128 * 10240 // (4 * requests * new * heads)))
        longest = _log_int(rng, min(most, 200), most)
        c = _decode("", requests, new, heads, rng.choice((128, 256, 512, 512)), rng.choice((32, 64, 64)), rng.choice((8, 12, 16, 16, 32, 64)),
                    max(new, longest // rng.choice((1, 4, 50))), longest, rng.choice((0, 0, 1)) if requests > 1 else 0, wide)
    elif op == "verify":
        requests, drafts = _log_int(rng, 1, 64), rng.choice((1, 2, 3, 5, 7, 10))
        c = _verify("", requests, drafts, _log_int(rng, 1000, min(200000, 64 * 3 * 131075 // (requests * drafts))), rng.random() < 0.5,
                    rng.random() < 0.7, rng.choice((0.6, 0.8, 1.0, 1.2)), rng.choice((1.0, 2.0, 4.0)), rng.choice(("bf16", "fp16", "fp32")))
    else:
        layers, block = _log_int(rng, 1, 60), rng.choice((8, 12, 16, 16, 32, 64))
        width, dtype = rng.choice((160, 320, 560, 576, 576, 583)), rng.choice(("bf16", "fp16", "e4m3"))
        pairs = _log_int(rng, 1, min(2000, 24 * 640 * 16 * 576 // (layers * block * width)))
        c = _copy("", layers, 2 * pairs + rng.randint(1, 500), pairs, block, width, rng.random() < 0.5, rng.choice((0, 0, pairs // 7)), dtype)
    del c["name"]
    return c


def _lengths(case):
    """Every request's new tokens and its cached ones with them, by the case alone."""
    rng = random.Random("%s" % sorted((k, v) for k, v in case.items() if k != "name"))
    n = case["requests"]
    spread = [_log_int(rng, case["shortest"], case["longest"]) for _ in range(n)]
    spread[0] = case["longest"]
    if case["op"] == "append":
        return spread, [x + rng.randint(0, case["cached"]) for x in spread]
    for i in range(case["empty"]):
        spread[n - 1 - 2 * i] = 0
    return [case["new"]] * n, spread


def _blocks(case, g, lengths):
    """(table, how many blocks): every request's blocks anywhere in the cache."""
    need = [-(-x // case["block"]) for x in lengths]
    blocks, first = sum(need) + 3, 0
    order = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(need), max(need), device="cuda", dtype=torch.int32)
    for b, k in enumerate(need):
        table[b, :k] = order[first:first + k]
        first += k
    return table, blocks


def _scale_for(largest):
    """The smallest power of two that brings the largest magnitude to the 8-bit type's range, in [2^-60, 2^60]."""
    fraction, exponent = torch.frexp((largest.double() / LARGEST).clamp_min(2.0 ** -60))
    return torch.ldexp(torch.ones_like(fraction), (exponent - (fraction == 0.5).to(exponent.dtype)).clamp(max=60)).float()


def _filled(case, g, blocks):
    """A cache of `blocks` blocks as appends leave it, tokens of different size among them, and its scales."""
    rank, width = case["rank"], case["rank"] + case["rot"]
    cache = torch.empty(blocks, case["block"], width, device="cuda", dtype=torch.float8_e4m3fn)
    scales = torch.empty(blocks, 2, device="cuda")
    step = max(1, (1 << 26) // (case["block"] * width))
    for at in range(0, blocks, step):
        n = min(step, blocks - at)
        x = torch.randn(n, case["block"], width, generator=g, device="cuda")
        x *= torch.exp(0.5 * torch.randn(n, case["block"], 1, generator=g, device="cuda"))
        x[..., rank:] *= 3.0
        s = _scale_for(torch.stack((x[..., :rank].abs().amax((1, 2)), x[..., rank:].abs().amax((1, 2))), 1))
        x[..., :rank] /= s[:, 0, None, None]
        x[..., rank:] /= s[:, 1, None, None]
        cache[at:at + n], scales[at:at + n] = x.to(cache.dtype), s
    return cache, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, op = TYPES[case["dtype"]], case["op"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    s = {"case": case}
    if op == "append":
        new, lengths = _lengths(case)
        s["table"], blocks = _blocks(case, g, lengths)
        s["cache"], s["scales"] = _filled(case, g, blocks)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["offsets"] = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda")
        s["latent"], s["key"] = normal(sum(new), case["rank"]), 3 * normal(sum(new), case["rot"])
        s["frequencies"] = (10000.0 ** (-torch.arange(case["rot"] // 2, dtype=torch.float64) * 2 / case["rot"])).cuda()
    elif op == "decode":
        _, lengths = _lengths(case)
        width = case["rank"] + case["rot"]
        s["table"], blocks = _blocks(case, g, lengths)
        s["cache"], s["scales"] = _filled(case, g, blocks)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["q"] = normal(len(lengths), case["new"], case["heads"], width)
        s["out"] = torch.empty(len(lengths), case["new"], case["heads"], case["rank"], device="cuda", dtype=dt)
        s["lse"] = torch.empty(len(lengths), case["new"], case["heads"], device="cuda")
        s["scale"] = 1.0 / math.sqrt(width)
    elif op == "verify":
        n, d, v = case["requests"], case["drafts"], case["vocab"]
        s["target"] = torch.randn(n, d + 1, v, generator=g, device="cuda") * case["spread"]
        guess = s["target"][:, :d] + 0.4 * torch.randn(n, d, v, generator=g, device="cuda")
        s["target"][..., ::97] = -math.inf  # tokens that a grammar rules out
        s["target"], guess = s["target"].to(dt), guess.to(dt)
        s["temperature"] = torch.full((n,), case["temperature"], device="cuda")
        if not case["known"]:  # the likeliest token of another model, as a text that repeats gives it
            s["tokens"], s["draft"] = guess.argmax(-1), None
            s["temperature"][::5] = 0.0
        else:  # drawn from the draft's distribution
            noise = torch.rand(guess.shape, generator=g, device="cuda").clamp_(1e-30, 1 - 1e-7)
            s["tokens"], s["draft"] = (guess.float() / case["temperature"] - torch.log(-torch.log(noise))).argmax(-1), guess
        s["uniform"] = torch.rand(n, d + 1, generator=g, device="cuda")
        s["drafted"] = torch.randint(0, d + 1, (n,), generator=g, device="cuda", dtype=torch.int32) if case["ragged"] else None
        s["out"] = torch.empty(n, d + 1, device="cuda", dtype=torch.int64)
        s["count"] = torch.empty(n, device="cuda", dtype=torch.int32)
        s["logprob"] = torch.empty(n, d + 1, device="cuda")
    else:
        shape = (case["layers"], case["blocks"], case["block"], case["width"])
        s["source"] = torch.empty(shape, device="cuda", dtype=dt)
        for layer in s["source"]:
            layer.copy_(torch.randn(shape[1:], generator=g, device="cuda"))
        order, n = torch.randperm(case["blocks"], generator=g, device="cuda").to(torch.int32), case["pairs"]
        s["from_blocks"], s["to_blocks"] = order[:n].clone(), order[n:2 * n].clone()
        if not case["inside"]:
            s["to_blocks"] = torch.randperm(case["blocks"], generator=g, device="cuda").to(torch.int32)[:n].clone()
        s["to_blocks"][n - case["padding"]:] = -1
        s["destination"] = s["source"] if case["inside"] else torch.zeros_like(s["source"])
    return s


def _turned(x, positions, frequencies, layout):
    """x [n, rot] in 32 bits, rotated.  The angle is reduced in 64 bits: 32 do not hold position times frequency."""
    angle = torch.remainder(positions.double()[:, None] * frequencies, 2 * math.pi).float()
    c, s = torch.cos(angle), torch.sin(angle)
    if layout == "half":
        a, b = x.chunk(2, -1)
        return torch.cat((a * c - b * s, a * s + b * c), -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)


def _plain_append(s):
    case, cache, scales = s["case"], s["cache"], s["scales"]
    rank, block = case["rank"], case["block"]
    n = s["latent"].shape[0]
    request = torch.searchsorted(s["offsets"], torch.arange(n, device="cuda", dtype=torch.int32), right=True) - 1
    position = s["lengths"][request] - s["offsets"][request + 1] + torch.arange(n, device="cuda")
    at, row = s["table"][request, position // block].long(), position % block
    key = _turned(s["key"].float(), position, s["frequencies"], case["layout"])
    latent = s["latent"].float()
    # every block's largest magnitudes and its first written row
    blocks = cache.shape[0]
    largest = torch.zeros(blocks, 2, device="cuda")
    first = torch.full((blocks,), block, device="cuda", dtype=torch.int64)
    for part, x in ((0, latent), (1, key)):
        largest[:, part].scatter_reduce_(0, at, x.abs().amax(1), "amax")
    first.scatter_reduce_(0, at, row, "amin")
    touched = torch.unique(at)
    first, before = first[touched], scales[touched]
    scale = _scale_for(largest[touched])
    scale = torch.where(first[:, None] == 0, scale, torch.maximum(scale, before))
    ratio = (before / scale).repeat_interleave(torch.tensor([rank, case["rot"]], device="cuda"), 1)
    held = cache[touched]
    old = torch.arange(block, device="cuda") < first[:, None]
    again = (held.float() * ratio[:, None, :]).to(cache.dtype)
    cache[touched] = torch.where(old[:, :, None], again.float(), held.float()).to(cache.dtype)
    scales[touched] = scale
    cache[at, row] = torch.cat((latent / scales[at, 0:1], key / scales[at, 1:2]), 1).to(cache.dtype)
    return cache, scales


def _plain_decode(s):
    case = s["case"]
    n, block, rank = s["table"].shape[1] * case["block"], case["block"], case["rank"]
    rows = s["cache"][s["table"].long()].float()  # [requests, blocks, block, width]
    scales = s["scales"][s["table"].long()]
    rows[..., :rank] *= scales[..., 0, None, None]
    rows[..., rank:] *= scales[..., 1, None, None]
    rows = rows.flatten(1, 2)
    at, new = torch.arange(n, device="cuda"), torch.arange(case["new"], device="cuda")
    seen = at[None, None, :] < (s["lengths"][:, None] - case["new"] + 1 + new)[:, :, None]
    scores = torch.matmul(s["q"].float().flatten(1, 2), rows.transpose(1, 2)).unflatten(1, (case["new"], -1)) * s["scale"]
    scores = scores.masked_fill(~seen[:, :, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    lse = (torch.log(total) + top).squeeze(-1)
    out = torch.matmul((e / total.clamp_min(1e-30)).flatten(1, 2), rows[..., :rank]).unflatten(1, (case["new"], -1))
    return out.to(s["q"].dtype), lse


def _plain_verify(s):
    """In 64 bits: the tokens are whole numbers, decided by sums over the vocabulary."""
    n, d, v = s["case"]["requests"], s["case"]["drafts"], s["case"]["vocab"]
    t = s["temperature"].double()[:, None, None]

    def probabilities(logits):
        x = logits.double()
        top = x.amax(-1, keepdim=True)
        w = torch.exp((x - top) / torch.where(t > 0, t, torch.ones_like(t)))
        place = torch.arange(v, device="cuda")
        first = torch.where(x == top, place, v).amin(-1, keepdim=True)
        w = torch.where(t > 0, w, (place == first).double())
        return w / w.sum(-1, keepdim=True)

    p = probabilities(s["target"])
    index = s["tokens"][..., None]
    real = torch.arange(d, device="cuda") < (torch.full((n,), d, device="cuda") if s["drafted"] is None else s["drafted"])[:, None]
    if s["draft"] is None:
        chance, drafted = torch.ones(n, d, device="cuda", dtype=torch.float64), None
    else:
        drafted = probabilities(s["draft"])
        chance = drafted.gather(2, index)[..., 0]
    passed = real & (s["uniform"][:, :d].double() * chance < p[:, :d].gather(2, index)[..., 0])
    accepted = passed.long().cumprod(1).sum(1)
    refused = accepted < real.sum(1)
    row = torch.arange(n, device="cuda")
    end = p[row, accepted]
    at = accepted.clamp(max=d - 1)
    other = torch.zeros_like(end).scatter_(1, s["tokens"][row, at][:, None], 1.0) if drafted is None else drafted[row, at]
    rest = (end - other).clamp_min(0)
    rest = torch.where((refused & (rest.sum(1) > 0))[:, None], rest, end)
    mass = rest.cumsum(1)
    token = torch.searchsorted(mass, s["uniform"][:, d:].double() * mass[:, -1:], right=True)
    place = torch.arange(d + 1, device="cuda")
    out = torch.cat((s["tokens"], token), 1)
    out = torch.where(place == accepted[:, None], token, torch.where(place < accepted[:, None], out, torch.full_like(out, -1)))
    logprob = torch.log(p.gather(2, out.clamp_min(0)[..., None])[..., 0]).float()
    return out, (accepted + 1).int(), logprob.masked_fill(out < 0, -math.inf)


def _plain_copy(s):
    kept = s["to_blocks"] >= 0
    s["destination"][:, s["to_blocks"][kept].long()] = s["source"][:, s["from_blocks"][kept].long()]
    return s["destination"]


def _own(s):
    from paper_2608_16336_gb300 import instance_ops as ops

    case = s["case"]
    op = case["op"]
    if op == "append":
        return ops.quantized_append(s["latent"], s["key"], s["frequencies"], s["offsets"], s["table"], s["lengths"], s["cache"], s["scales"],
                                    layout=case["layout"])
    if op == "decode":
        return ops.quantized_decode(s["q"], s["cache"], s["scales"], s["table"], s["lengths"], scale=s["scale"], out=s["out"], lse=s["lse"])
    if op == "verify":
        return ops.verify(s["target"], s["tokens"], s["uniform"], draft=s["draft"], temperature=s["temperature"], drafted=s["drafted"],
                          out=s["out"], count=s["count"], logprob=s["logprob"])
    return ops.block_copy(s["source"], s["destination"], s["from_blocks"], s["to_blocks"])


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "decode": _plain_decode, "verify": _plain_verify, "copy": _plain_copy}[state["case"]["op"]](state)


def work(case):
    e, op = SIZE[case["dtype"]], case["op"]
    if op == "append":
        new, lengths = _lengths(case)
        n, width = sum(new), case["rank"] + case["rot"]
        blocks = sum(-(-k // case["block"]) - (k - q) // case["block"] for q, k in zip(new, lengths))
        return {"bytes": n * width * (e + 1) + 12 * blocks + 8 * len(new) + 4 * case["rot"], "flops": 3 * n * width}
    if op == "decode":
        q, k = _lengths(case)
        rows = sum(q) * case["heads"]
        width = case["rank"] + case["rot"]
        pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(q, k) if b)
        return {"bytes": sum(k) * width + 12 * sum(-(-x // case["block"]) for x in k) + e * rows * (width + case["rank"]) + 4 * rows,
                "flops": 2 * case["heads"] * pairs * (width + case["rank"])}
    if op == "verify":
        rows = case["requests"] * (2 * case["drafts"] + 1 if case["known"] else case["drafts"] + 1)
        return {"bytes": rows * case["vocab"] * e + case["requests"] * (24 * case["drafts"] + 24), "flops": 4 * rows * case["vocab"]}
    n = case["pairs"] - case["padding"]
    return {"bytes": 2 * n * case["layers"] * case["block"] * case["width"] * e + 8 * case["pairs"], "flops": 0}


def _to_8_bits(x):
    """The nearest numbers with four significant bits, multiples of 2^-9 at least, ties to the even one."""
    size = x.abs().clamp_min(2.0 ** -6)
    step = torch.exp2(torch.floor(torch.log2(size)) - 3)
    return torch.round(x / step) * step


def _exact_append(s):
    case, cache, scales = s["case"], s["cache"].double(), s["scales"].double()
    new, lengths = _lengths(case)
    rank, block, table = case["rank"], case["block"], s["table"].tolist()
    ids, starts, rows, at = [], [], [], 0
    for b, (n, end) in enumerate(zip(new, lengths)):  # (block, first row, rows) of every block that a request writes
        for i in range((end - n) // block, -(-end // block)):
            lo, hi = max(end - n, i * block), min(end, (i + 1) * block)
            ids.append(table[b][i]), starts.append((lo - i * block, at + lo - (end - n))), rows.append(hi - lo)
        at += n
    position = torch.cat([torch.arange(end - n, end) for n, end in zip(new, lengths)]).cuda().double()
    z = torch.polar(torch.ones_like(s["frequencies"]), torch.remainder(position[:, None] * s["frequencies"], 2 * math.pi))
    half = case["rot"] // 2
    pair = (s["key"][:, :half], s["key"][:, half:]) if case["layout"] == "half" else (s["key"][:, ::2], s["key"][:, 1::2])
    y = torch.complex(pair[0].double().contiguous(), pair[1].double().contiguous()) * z
    key = torch.cat((y.real, y.imag), 1) if case["layout"] == "half" else torch.view_as_real(y).flatten(1)
    x = torch.cat((s["latent"].double(), key), 1)
    # the written rows of every block side by side, the others left out by their number
    ids, rows = torch.tensor(ids, device="cuda"), torch.tensor(rows, device="cuda")
    first, source = (torch.tensor(v, device="cuda") for v in zip(*starts))
    place = torch.arange(block, device="cuda")
    written = (place >= first[:, None]) & (place < (first + rows)[:, None])
    wanted = x[(source[:, None] + place - first[:, None]).clamp(0, x.shape[0] - 1)] * written[:, :, None]
    held = cache[ids]
    for part, cols in ((0, slice(0, rank)), (1, slice(rank, None))):
        most = wanted[..., cols].abs().amax((1, 2))
        scale = torch.exp2(torch.ceil(torch.log2(most / LARGEST)).clamp(-60, 60))
        scale = torch.where(first > 0, torch.maximum(scale, scales[ids, part]), scale)
        kept = _to_8_bits(held[..., cols] * (scales[ids, part] / scale)[:, None, None])
        fresh = _to_8_bits(wanted[..., cols] / scale[:, None, None])
        cache[ids, :, cols] = torch.where(written[:, :, None], fresh, torch.where((place < first[:, None])[:, :, None], kept, held[..., cols]))
        scales[ids, part] = scale
    return cache, scales


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "append":
        return _exact_append(s)
    if op == "decode":
        new, lengths = _lengths(case)
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lengths):
            blocks = s["table"][b, :-(-n // case["block"])].long()
            part = s["scales"][blocks].double()
            row = s["cache"][blocks].double()
            row = torch.cat((row[..., :case["rank"]] * part[:, :1, None], row[..., case["rank"]:] * part[:, 1:, None]), 2).flatten(0, 1)[:n]
            for t in range(new[b]):
                m = n - new[b] + 1 + t
                if m > 0:
                    x = s["q"][b, t].double() @ row[:m].T * s["scale"]
                    lse[b, t] = torch.logsumexp(x, 1)
                    out[b, t] = torch.exp(x - lse[b, t][:, None]) @ row[:m, :case["rank"]]
        return out, lse
    if op == "verify":
        d, v = case["drafts"], case["vocab"]
        out, count, logprob = [], [], []
        for b in range(case["requests"]):
            t = float(s["temperature"][b])

            def logs(row):
                if t > 0:
                    return torch.log_softmax(row.double() / t, 0)
                first = int((row == row.max()).nonzero()[0])
                return torch.full((v,), -math.inf, dtype=torch.float64, device="cuda").index_fill_(0, torch.tensor([first], device="cuda"), 0.0)

            tokens, lps, u = [], [], s["uniform"][b].double().tolist()
            drafted = d if s["drafted"] is None else int(s["drafted"][b])
            for i in range(drafted + 1):
                p = logs(s["target"][b, i])
                weight = torch.exp(p)
                if i < drafted:
                    x = int(s["tokens"][b, i])
                    if s["draft"] is None:
                        q = torch.zeros(v, dtype=torch.float64, device="cuda")
                        q[x] = 1.0
                    else:
                        q = torch.exp(logs(s["draft"][b, i]))
                    if u[i] * float(q[x]) < float(weight[x]):
                        tokens.append(x), lps.append(float(p[x]))
                        continue
                    over = torch.relu(weight - q)
                    weight = over if float(over.sum()) > 0 else weight
                sums = torch.cumsum(weight, 0)
                x = int((sums <= u[d] * sums[-1]).sum())
                tokens.append(x), lps.append(float(p[x]))
                break
            left = d + 1 - len(tokens)
            out.append(tokens + [-1] * left), count.append(len(tokens)), logprob.append(lps + [-math.inf] * left)
        return (torch.tensor(out), torch.tensor(count, dtype=torch.int32), torch.tensor(logprob, dtype=torch.float64))
    return None  # copied numbers
