"""Performance cases of an instance's iteration operators.

The simulator's instances keep their requests' keys and values in blocks of T
tokens and run iterations of prefills and single tokens.  These cases time
the operators of such an iteration on the device:

* ``rotary``: rotary positions on part of every head;
* ``append``: a token's latent vector and rotated shared key into the blocks;
* ``decode``: attention of new tokens over the block cache, queries already
  in the latent space (the absorbed form);
* ``prefill``: causal attention of ragged prompts with expanded keys and
  values, after a cached prefix or none;
* ``sample``: the next token under temperature, top-k, top-p and min-p from
  given uniform numbers.

A case's lengths come from the case alone and its values from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}


def _rotary(name, tokens, heads, dim, rot, offset, layout, dtype, span, ramp=False):
    return dict(name=name, op="rotary", tokens=tokens, heads=heads, dim=dim, rot=rot, offset=offset, layout=layout,
                dtype=dtype, span=span, ramp=ramp)


def _append(name, tokens, rank, rot, block, blocks, layout, dtype, span):
    return dict(name=name, op="append", tokens=tokens, rank=rank, rot=rot, block=block, blocks=blocks, layout=layout,
                dtype=dtype, span=span)


def _decode(name, requests, new, heads, rank, rot, block, shortest, longest, empty, dtype):
    return dict(name=name, op="decode", requests=requests, new=new, heads=heads, rank=rank, rot=rot, block=block,
                shortest=shortest, longest=longest, empty=empty, dtype=dtype)


def _prefill(name, requests, heads, nope, rot, value, shortest, longest, prefix, dtype):
    return dict(name=name, op="prefill", requests=requests, heads=heads, nope=nope, rot=rot, value=value,
                shortest=shortest, longest=longest, prefix=prefix, dtype=dtype)


def _sample(name, rows, vocab, top_k, top_p, min_p, spread, dtype):
    return dict(name=name, op="sample", rows=rows, vocab=vocab, top_k=top_k, top_p=top_p, min_p=min_p, spread=spread,
                dtype=dtype)


def listed():
    return [
        # one iteration of a full running batch, 64 single tokens: latency of a small launch
        _rotary("rotary_batch", 64, 16, 192, 64, 128, "interleaved", "bf16", 8192),
        # the queries of a large prefill, positions past the trained context with ramped frequencies
        _rotary("rotary_prompts", 8192, 128, 192, 64, 128, "half", "bf16", 131072, True),
        # the same batch's 64 new rows into an instance of 2,048 blocks
        _append("append_batch", 64, 512, 64, 16, 2048, "interleaved", "bf16", 8192),
        # a prefill of 20,011 tokens into scattered blocks of 12, some rows being padding
        _append("append_prompts", 20011, 512, 64, 12, 4096, "half", "fp16", 16384),
        # one lightly loaded request with a short context
        _decode("decode_one", 1, 1, 16, 512, 64, 16, 777, 777, 0, "bf16"),
        # a full running batch with every head on this GPU, prompts as in the long-prompt traces, some slots empty
        _decode("decode_batch", 64, 1, 128, 512, 64, 16, 200, 10240, 3, "bf16"),
        # a few requests with very long contexts and two new tokens each
        _decode("decode_long", 3, 2, 16, 512, 64, 64, 90001, 130000, 0, "fp16"),
        # many short prompts admitted in one iteration
        _prefill("prefill_short", 37, 16, 128, 64, 128, 1, 300, 0, "fp16"),
        # chunks of prompts whose first part is in the cache already
        _prefill("prefill_chunk", 4, 32, 128, 64, 128, 450, 513, 4100, "bf16"),
        # one prompt of the traces' longest length
        _prefill("prefill_long", 1, 64, 128, 64, 128, 8192, 8192, 0, "bf16"),
        # one request's next token
        _sample("sample_one", 1, 32000, 50, 0.9, 0.02, 3.0, "fp32"),
        # the whole running batch, large vocabulary, nucleus without a bound on its size for most rows
        _sample("sample_batch", 64, 131075, 1000, 0.95, 0.0, 2.0, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi + 0.49))))))


def draw(rng):
    op = rng.choice(("rotary", "append", "decode", "prefill", "sample"))
    layout, wide = rng.choice(("interleaved", "half")), rng.choice(("bf16", "fp16"))
    if op == "rotary":
        rot = rng.choice((32, 64, 64, 96, 128))
        offset = rng.choice((0, 8, 64, 128))
        heads = _log_int(rng, 1, 128)
        c = _rotary("", _log_int(rng, 1, min(16384, 1048576 // heads)), heads, rot + offset + rng.choice((0, 0, 8)), rot, offset, layout,
                    rng.choice(("bf16", "fp16", "fp32")), _log_int(rng, 4096, 1000000), rng.random() < 0.4)
    elif op == "append":
        block = rng.choice((8, 12, 16, 16, 32, 64))
        tokens = _log_int(rng, 1, 32768)
        c = _append("", tokens, rng.choice((128, 256, 512, 512)), rng.choice((32, 64, 64)), block, -(-tokens // block) + rng.randint(8, 512),
                    layout, wide, _log_int(rng, 4096, 1000000))
    elif op == "decode":
        requests, new, heads = _log_int(rng, 1, 64), rng.choice((1, 1, 1, 2, 3, 5)), _log_int(rng, 1, 128)
        most = max(64, min(130000, 64 * 10240 // (2 * requests), 64 * 128 * 10240 // (4 * requests * new * heads)))
        longest = _log_int(rng, min(most, 200), most)
        c = _decode("", requests, new, heads, rng.choice((128, 256, 512, 512)), rng.choice((32, 64, 64)), rng.choice((8, 12, 16, 16, 32, 64)),
                    max(new, longest // rng.choice((1, 4, 50))), longest, rng.choice((0, 0, 1)) if requests > 1 else 0, wide)
    elif op == "prefill":
        requests, heads = _log_int(rng, 1, 64), _log_int(rng, 1, 64)
        longest = _log_int(rng, 48, int(8192 / math.sqrt(requests)))
        prefix = 0 if rng.random() < 0.6 else _log_int(rng, 1, 4096 if requests <= 4 else 512)
        heads = max(1, min(heads, int(64 * 8192 * 4096 / (requests * longest * (longest + prefix)))))
        c = _prefill("", requests, heads, rng.choice((64, 128, 128)), rng.choice((32, 64)), rng.choice((64, 128, 128)),
                     max(1, longest // rng.choice((1, 3, 40))), longest, prefix, wide)
    else:
        c = _sample("", _log_int(rng, 1, 256), _log_int(rng, 1000, 200000), rng.choice((0, 20, 200, 2000)), rng.choice((1.0, 0.9, 0.8)),
                    rng.choice((0.0, 0.0, 0.05)), rng.choice((1.0, 2.0, 4.0)), rng.choice(("bf16", "fp16", "fp32")))
    del c["name"]
    return c


def _lengths(case):
    """Every request's new tokens and context (a prefill: prompt and prompt with its prefix), by the case alone."""
    rng = random.Random("%s" % sorted((k, v) for k, v in case.items() if k != "name"))
    n = case["requests"]
    spread = [_log_int(rng, case["shortest"], case["longest"]) for _ in range(n)]
    spread[0] = case["longest"]
    if case["op"] == "prefill":
        return spread, [x + (rng.randint(0, case["prefix"]) if case["prefix"] else 0) for x in spread]
    for i in range(case["empty"]):
        spread[n - 1 - 2 * i] = 0
    return [case["new"]] * n, spread


def _frequencies(rot, ramp):
    """Radians per position of each pair; with `ramp`, the slow ones are slowed eight times more, the fast ones not."""
    f = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    if ramp:
        turns = 16384 * f / (2 * math.pi)
        f = f * (1 + (1 / 8 - 1) * ((32 - turns) / 31).clamp(0, 1))
    return f


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    s = {"case": case}
    if case["op"] in ("rotary", "append"):
        n = case["tokens"]
        s["positions"] = torch.randint(0, case["span"], (n,), generator=g, device="cuda", dtype=torch.int32)
        s["frequencies"] = _frequencies(case["rot"], case.get("ramp", False)).cuda()
    if case["op"] == "rotary":
        s["x"] = normal(n, case["heads"], case["dim"])
        s["out"] = torch.empty_like(s["x"])
        s["amplitude"] = 1.2079 if case["ramp"] else 1.0  # 0.1 ln 8 + 1
    elif case["op"] == "append":
        rows, block = case["blocks"] * case["block"], case["block"]
        s["latent"], s["key"] = normal(n, case["rank"]), normal(n, case["rot"])
        s["cache"] = torch.zeros(case["blocks"], block, case["rank"] + case["rot"], device="cuda", dtype=dt)
        at = torch.randperm(case["blocks"], generator=g, device="cuda")[:, None] * block + torch.arange(block, device="cuda")
        s["slots"] = at.reshape(rows)[:n].clone()
        s["slots"][torch.rand(n, generator=g, device="cuda") < 0.01] = -1  # padding
    elif case["op"] == "decode":
        _, lengths = _lengths(case)
        width, block = case["rank"] + case["rot"], case["block"]
        need = [-(-x // block) for x in lengths]
        blocks = sum(need) + 3
        order = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
        s["table"] = torch.zeros(len(need), max(need), device="cuda", dtype=torch.int32)
        first = 0
        for b, k in enumerate(need):
            s["table"][b, :k] = order[first:first + k]
            first += k
        s["cache"] = normal(blocks, block, width)
        s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        s["q"] = normal(len(lengths), case["new"], case["heads"], width)
        s["out"] = torch.empty(len(lengths), case["new"], case["heads"], case["rank"], device="cuda", dtype=dt)
        s["lse"] = torch.empty(len(lengths), case["new"], case["heads"], device="cuda")
        s["scale"] = 1.6 / math.sqrt(width)
    elif case["op"] == "prefill":
        q, k = _lengths(case)
        s["scale"] = 1.6 / math.sqrt(case["nope"] + case["rot"])
        s["longest"] = max(q)
        for name, n in (("q_offsets", q), ("k_offsets", k)):
            s[name] = torch.tensor(np.cumsum([0] + n), dtype=torch.int32, device="cuda")
        s["q"] = normal(sum(q), case["heads"], case["nope"] + case["rot"])
        s["key"] = normal(sum(k), case["heads"], case["nope"])
        s["shared"] = normal(sum(k), case["rot"])
        s["value"] = normal(sum(k), case["heads"], case["value"])
        s["out"] = torch.empty(sum(q), case["heads"], case["value"], device="cuda", dtype=dt)
        s["lse"] = torch.empty(sum(q), case["heads"], device="cuda")
    else:
        n = case["rows"]
        s["logits"] = (torch.randn(n, case["vocab"], generator=g, device="cuda") * case["spread"]).to(dt)
        s["logits"][:, ::97] = -math.inf  # tokens that a grammar rules out
        s["uniform"] = torch.rand(n, generator=g, device="cuda")

        def mixed(value, without, rare):
            """`value` for the rows that set it, `without` for those that do not."""
            return torch.where(torch.rand(n, generator=g, device="cuda") < rare, torch.full((n,), without, device="cuda"),
                               torch.full((n,), value, device="cuda"))

        s["temperature"] = mixed(0.8, 1.3, 0.3)
        s["top_k"] = mixed(float(case["top_k"]), 0.0, 0.7 if n > 1 else 0.0).to(torch.int32)
        s["top_p"] = mixed(case["top_p"], 1.0, 0.2 if n > 1 else 0.0)
        s["min_p"] = mixed(case["min_p"], 0.0, 0.5 if n > 1 else 0.0)
        s["token"] = torch.empty(n, device="cuda", dtype=torch.int64)
        s["logprob"] = torch.empty(n, device="cuda")
    return s


def _turned(x, positions, frequencies, layout, amplitude):
    """x [n, heads, rot] in 32 bits, rotated.  The angle is reduced in 64 bits: 32 do not hold position times frequency."""
    angle = torch.remainder(positions.double()[:, None] * frequencies, 2 * math.pi).float()[:, None, :]
    c, s = torch.cos(angle) * amplitude, torch.sin(angle) * amplitude
    if layout == "half":
        a, b = x.chunk(2, -1)
        return torch.cat((a * c - b * s, a * s + b * c), -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)


def _attended(scores, seen):
    """Softmax weights of the scores that are seen (none: zeros) and the logarithm of their sum."""
    scores = scores.masked_fill(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = torch.exp(scores - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return e / total.clamp_min(1e-30), (torch.log(total) + top).squeeze(-1)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "rotary":
        a, b = case["offset"], case["offset"] + case["rot"]
        y = s["x"].float()
        y[..., a:b] = _turned(y[..., a:b], s["positions"], s["frequencies"], case["layout"], s["amplitude"])
        return y.to(s["x"].dtype)
    if op == "append":
        key = _turned(s["key"].float()[:, None], s["positions"], s["frequencies"], case["layout"], 1.0)[:, 0].to(s["key"].dtype)
        kept = s["slots"] >= 0
        s["cache"].view(-1, s["cache"].shape[-1])[s["slots"][kept]] = torch.cat((s["latent"], key), -1)[kept]
        return s["cache"]
    if op == "decode":
        n, block = s["table"].shape[1] * case["block"], case["block"]
        rows = s["cache"][s["table"].long()].flatten(1, 2).float()  # [requests, n, width]
        at = torch.arange(n, device="cuda")
        new = torch.arange(case["new"], device="cuda")
        seen = at[None, None, :] < (s["lengths"][:, None] - case["new"] + 1 + new)[:, :, None]
        scores = torch.matmul(s["q"].float().flatten(1, 2), rows.transpose(1, 2)).unflatten(1, (case["new"], -1)) * s["scale"]
        p, lse = _attended(scores, seen[:, :, None, :])
        out = torch.matmul(p.flatten(1, 2), rows[..., :case["rank"]]).unflatten(1, (case["new"], -1))
        return out.to(s["q"].dtype), lse
    if op == "prefill":
        nq, nk = (s["q_offsets"].diff().long(), s["k_offsets"].diff().long())
        most_q, most_k = s["longest"], s["longest"] + case["prefix"]
        at_q, at_k = torch.arange(most_q, device="cuda"), torch.arange(most_k, device="cuda")
        rows_q, rows_k = s["q_offsets"][:-1, None] + at_q, s["k_offsets"][:-1, None] + at_k
        real_q, real_k = at_q < nq[:, None], at_k < nk[:, None]
        rows_q, rows_k = rows_q.clamp(max=s["q"].shape[0] - 1), rows_k.clamp(max=s["key"].shape[0] - 1)
        q = s["q"].float()[rows_q].transpose(1, 2)  # [requests, heads, rows, width]
        key = s["key"].float()[rows_k].transpose(1, 2)
        scores = torch.matmul(q[..., :case["nope"]], key.transpose(2, 3))
        scores += torch.matmul(q[..., case["nope"]:], s["shared"].float()[rows_k].transpose(1, 2)[:, None])
        scores *= s["scale"]
        seen = real_k[:, None, :] & (at_k <= at_q[:, None] + (nk - nq)[:, None, None])
        p, lse = _attended(scores, seen[:, None])
        out = torch.matmul(p, s["value"].float()[rows_k].transpose(1, 2)).transpose(1, 2)
        return out[real_q].to(s["q"].dtype), lse.transpose(1, 2)[real_q]
    # sampling: sorted by descending logit (ties: lowest index first); sums in 64 bits, as the token is a whole number
    logits = s["logits"].float()
    v = logits.shape[1]
    value, order = torch.sort(logits, dim=1, descending=True, stable=True)
    w = torch.exp((value - value[:, :1]) / s["temperature"][:, None])
    k = torch.where(s["top_k"] > 0, s["top_k"], v)
    kept = torch.arange(v, device="cuda") < k[:, None]
    mass = torch.cumsum((w * kept).double(), 1)
    kept &= (mass - w) < s["top_p"][:, None].double() * mass[:, -1:]
    kept &= w >= s["min_p"][:, None]
    drawn = torch.zeros_like(w).scatter_(1, order, w * kept)  # back in vocabulary order
    mass = torch.cumsum(drawn.double(), 1)
    token = torch.searchsorted(mass, s["uniform"][:, None].double() * mass[:, -1:], right=True)
    logprob = torch.log(drawn.gather(1, token)) - torch.log(mass[:, -1:]).float()
    return token[:, 0], logprob[:, 0]


def _own(s):
    from paper_2608_16336_gb300 import instance_ops as ops

    case = s["case"]
    op = case["op"]
    if op == "rotary":
        return ops.rotary(s["x"], s["positions"], s["frequencies"], layout=case["layout"], offset=case["offset"],
                          amplitude=s["amplitude"], out=s["out"])
    if op == "append":
        return ops.latent_append(s["latent"], s["key"], s["positions"], s["frequencies"], s["slots"], s["cache"],
                                 layout=case["layout"])
    if op == "decode":
        return ops.latent_decode(s["q"], s["cache"], s["table"], s["lengths"], scale=s["scale"], out=s["out"], lse=s["lse"])
    if op == "prefill":
        return ops.latent_prefill(s["q"], s["key"], s["shared"], s["value"], s["q_offsets"], s["k_offsets"], scale=s["scale"],
                                  longest=s["longest"], out=s["out"], lse=s["lse"])
    return ops.sample(s["logits"], s["uniform"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                      min_p=s["min_p"], out=s["token"], logprob=s["logprob"])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    e, op = SIZE[case["dtype"]], case["op"]
    if op == "rotary":
        n = case["tokens"] * case["heads"]
        return {"bytes": 2 * n * case["dim"] * e + 4 * case["tokens"] + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    if op == "append":
        n, width = case["tokens"], case["rank"] + case["rot"]
        return {"bytes": 2 * n * width * e + 12 * n + 4 * case["rot"], "flops": 3 * n * case["rot"]}
    if op == "decode":
        q, k = _lengths(case)
        rows = sum(q) * case["heads"]
        width = case["rank"] + case["rot"]
        pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(q, k) if b)
        return {"bytes": e * (sum(k) * width + rows * (width + case["rank"])) + 4 * (rows + sum(-(-x // case["block"]) for x in k)),
                "flops": 2 * case["heads"] * pairs * (width + case["rank"])}
    if op == "prefill":
        q, k = _lengths(case)
        h, width = case["heads"], case["nope"] + case["rot"]
        pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(q, k))
        return {"bytes": e * (sum(q) * h * (width + case["value"]) + sum(k) * (h * (case["nope"] + case["value"]) + case["rot"])) + 4 * sum(q) * h,
                "flops": 2 * h * pairs * (width + case["value"])}
    n = case["rows"] * case["vocab"]
    return {"bytes": n * e + 32 * case["rows"], "flops": 4 * n}


def _exact_turn(x, positions, frequencies, layout, amplitude):
    """Complex multiplication by amplitude * exp(i * position * frequency)."""
    z = amplitude * torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), torch.remainder(positions.double()[:, None] * frequencies, 2 * math.pi))
    half = x.shape[-1] // 2
    pair = (x[..., :half], x[..., half:]) if layout == "half" else (x[..., ::2], x[..., 1::2])
    y = torch.complex(pair[0].contiguous(), pair[1].contiguous()) * z.reshape(z.shape[:1] + (1,) * (x.dim() - 2) + z.shape[1:])
    return torch.cat((y.real, y.imag), -1) if layout == "half" else torch.view_as_real(y).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rotary":
        y = s["x"].double()
        part = y.narrow(-1, case["offset"], case["rot"])
        part.copy_(_exact_turn(part.clone(), s["positions"], s["frequencies"], case["layout"], s["amplitude"]))
        return y
    if op == "append":
        cache = s["cache"].double()
        key = _exact_turn(s["key"].double(), s["positions"], s["frequencies"], case["layout"], 1.0)
        kept = torch.nonzero(s["slots"] >= 0)[:, 0]
        block, row = s["slots"][kept] // case["block"], s["slots"][kept] % case["block"]
        cache[block, row, :case["rank"]] = s["latent"][kept].double()
        cache[block, row, case["rank"]:] = key[kept]
        return cache
    if op == "decode":
        new, lengths = _lengths(case)
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lengths):
            blocks = s["table"][b, :-(-n // case["block"])].long()
            row = s["cache"][blocks].reshape(-1, s["cache"].shape[-1])[:n].double()
            for t in range(new[b]):
                m = n - new[b] + 1 + t
                if m > 0:
                    x = s["q"][b, t].double() @ row[:m].T * s["scale"]
                    lse[b, t] = torch.logsumexp(x, 1)
                    out[b, t] = torch.exp(x - lse[b, t][:, None]) @ row[:m, :case["rank"]]
        return out, lse
    if op == "prefill":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        q_at, k_at = s["q_offsets"].tolist(), s["k_offsets"].tolist()
        for q0, q1, k0, k1 in zip(q_at, q_at[1:], k_at, k_at[1:]):
            hidden = torch.ones(q1 - q0, k1 - k0, dtype=torch.bool, device="cuda").triu(k1 - k0 - (q1 - q0) + 1)
            for h in range(case["heads"]):
                key = torch.cat((s["key"][k0:k1, h], s["shared"][k0:k1]), 1).double()
                x = (s["q"][q0:q1, h].double() @ key.T * s["scale"]).masked_fill_(hidden, -math.inf)
                lse[q0:q1, h] = torch.logsumexp(x, 1)
                out[q0:q1, h] = torch.softmax(x, 1) @ s["value"][k0:k1, h].double()
        return out, lse
    logits = s["logits"].double().cpu().numpy()
    u, temperature, top_k, top_p, min_p = (s[k].double().cpu().numpy() for k in ("uniform", "temperature", "top_k", "top_p", "min_p"))
    token, logprob = [], []
    for b, row in enumerate(logits):
        w = np.exp((row - row.max()) / temperature[b])
        best = np.argsort(-row, kind="stable")
        if top_k[b] > 0:
            best = best[:int(top_k[b])]
        mass = np.cumsum(w[best])
        best = best[:1 + int(np.searchsorted(mass, top_p[b] * mass[-1], side="left"))]
        best = np.sort(best[w[best] >= min_p[b]])
        mass = np.cumsum(w[best])
        token.append(int(best[min(int(np.searchsorted(mass, u[b] * mass[-1], side="right")), len(best) - 1)]))
        logprob.append(math.log(w[token[-1]] / mass[-1]))
    return np.array(token), np.array(logprob)
