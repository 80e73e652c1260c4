"""The iteration's operators on the GPU against their formulas in 64 bits, at
the sizes, strides and masks where they can go wrong.

Tolerances, per element, from the arithmetic: a result rounded once to a type
of unit roundoff u / 2 (bfloat16: u = 2^-8) is off by less than u |y|; attention weights rounded to that type add at most u sum_j p_j |v_j|
(2 u is allowed); 32-bit arithmetic adds 1e-5 of the same sum (a
score of 576 products is good to about 1e-6 of their absolute sum)."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF: 2.0 ** -8, HF: 2.0 ** -11, F32: 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    yield
    assert ops.faults() == 0  # no wait inside a kernel ran out


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


# ------------------------------------------------------------- rotary -----
def turned(x, pos, freq, layout, amplitude=1.0, sign=1):
    """x [n, ..., rot] in 64 bits as complex numbers; angles reduced in integers of 2^-64 turns, on the host."""
    turns = [round(f / (2 * math.pi) * 2 ** 64) for f in freq.double().tolist()]
    angle = torch.tensor([[(p * t % 2 ** 64) / 2 ** 64 * 2 * math.pi for t in turns] for p in pos.tolist()], dtype=torch.float64)
    z = amplitude * torch.exp(1j * sign * angle).cuda().reshape((x.shape[0],) + (1,) * (x.dim() - 2) + (-1,))
    half = x.shape[-1] // 2
    x = x.double()
    a, b = (x[..., :half], x[..., half:]) if layout == "half" else (x[..., 0::2], x[..., 1::2])
    y = torch.complex(a.contiguous(), b.contiguous()) * z
    return torch.cat((y.real, y.imag), -1) if layout == "half" else torch.stack((y.real, y.imag), -1).flatten(-2)


def check_rotary(x, pos, freq, got, layout, offset, amplitude=1.0, sign=1):
    rot = 2 * freq.shape[0]
    want = x.double()
    want[..., offset:offset + rot] = turned(x[..., offset:offset + rot], pos, freq, layout, amplitude, sign)
    part = got.double()[..., offset:offset + rot] - want[..., offset:offset + rot]
    w = want[..., offset:offset + rot]
    # a pair's rounding in 32 bits goes by the pair's length: |a| + |b| <= 2 max
    size = x.double()[..., offset:offset + rot].abs().amax(-1, keepdim=True) * abs(amplitude)
    assert (part.abs() <= U[x.dtype] * w.abs() + 2e-6 * size).all(), float(part.abs().max())
    keep = torch.ones(x.shape[-1], dtype=torch.bool)
    keep[offset:offset + rot] = False
    assert torch.equal(got[..., keep], x[..., keep])


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("tokens,heads,dim,rot,offset", [
    (1, 1, 2, 2, 0), (3, 5, 7, 4, 1), (64, 16, 192, 64, 128), (17, 3, 64, 64, 0), (5, 2, 100, 96, 3), (9, 1, 256, 256, 0),
    (33, 40, 130, 128, 2), (700, 7, 72, 32, 40), (2, 300, 64, 10, 20)])
def test_rotary(tokens, heads, dim, rot, offset, dtype, layout):
    g = gen(tokens * 1000 + heads)
    x = randn(g, tokens, heads, dim, dtype=dtype)
    pos = torch.randint(0, 100000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    f = ops.rotary_frequencies(rot)
    y = ops.rotary(x, pos, f, layout=layout, offset=offset)
    check_rotary(x, pos, f, y, layout, offset)
    z = x.clone()
    assert ops.rotary(z, pos, f, layout=layout, offset=offset, out=z) is z
    assert torch.equal(z, y)  # in place: the same bits
    assert torch.equal(ops.rotary(x, pos.long(), f, layout=layout, offset=offset), y)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tokens,heads,dim,rot,offset", [(20011, 1, 32, 32, 0), (3001, 12, 104, 96, 8), (5000, 10, 160, 32, 64), (2500, 1, 512, 256, 0),
                                                         (1300, 300, 64, 32, 16)])
def test_rotary_many_tokens(tokens, heads, dim, rot, offset, dtype, layout):
    """Groups of tokens a block, the last one short; nothing past the last token is written."""
    g = gen(tokens)
    x = randn(g, tokens, heads, dim, dtype=dtype)
    pos = torch.randint(0, 100000, (tokens,), generator=g, device="cuda")
    f = ops.rotary_frequencies(rot)
    store = torch.full((tokens + 3, heads, dim), 7.0, device="cuda", dtype=dtype)
    y = ops.rotary(x, pos, f, layout=layout, offset=offset, out=store[:tokens])
    check_rotary(x, pos, f, y, layout, offset)
    assert (store[tokens:] == 7.0).all()
    store[:tokens] = x
    ops.rotary(store[:tokens], pos, f, layout=layout, offset=offset, out=store[:tokens])
    assert torch.equal(store[:tokens], ops.rotary(x, pos, f, layout=layout, offset=offset)) and (store[tokens:] == 7.0).all()


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_rotary_positions_far_out(layout):
    g = gen(1)
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 40 + 12345, -2 ** 62, 10 ** 15, 7], device="cuda")
    x = randn(g, len(pos), 2, 64)
    f = ops.rotary_frequencies(64, scaling="ramp", factor=8.0, trained=4096)
    y = ops.rotary(x, pos, f, layout=layout, amplitude=ops.ramp_amplitude(8.0))
    # the frequency itself is a 64-bit float: its last bit is 2^-53 of a turn and the position multiplies it
    turns = f / (2 * math.pi)
    near = (pos.double()[:, None] * turns * 2.0 ** -52).abs().amax(1) < 1e-7
    check_rotary(x[near], pos[near], f, y[near], layout, 0, ops.ramp_amplitude(8.0))
    assert int(near.sum()) >= 6 and torch.isfinite(y).all()
    length = x.double().square().sum(-1) * ops.ramp_amplitude(8.0) ** 2  # a rotation at any position
    assert torch.allclose(y.double().square().sum(-1), length, rtol=1e-5)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_rotary_strides_and_alignment(layout, dtype):
    g = gen(2)
    pos = torch.arange(6, device="cuda", dtype=torch.int32) * 1001
    f = ops.rotary_frequencies(64)
    base = randn(g, 8 * 12 * 200 + 64, dtype=dtype)
    for first, strides in ((0, (12 * 200, 200, 1)), (3, (12 * 200, 200, 1)), (1, (200, 6 * 200, 1)), (8, (2001, 131, 1)), (0, (0, 128, 1))):
        x = base.as_strided((6, 4, 128), strides, first)
        for offset in (0, 5, 64):
            check_rotary(x, pos, f, ops.rotary(x, pos, f, layout=layout, offset=offset), layout, offset)
    out = torch.full((6, 9, 133), 7.0, device="cuda", dtype=dtype)
    view = out[:, 2:6, 3:131]
    ops.rotary(base.as_strided((6, 4, 128), (512, 128, 1)), pos, f, layout=layout, offset=64, out=view)
    check_rotary(base.as_strided((6, 4, 128), (512, 128, 1)), pos, f, view, layout, 64)
    view.fill_(7.0)
    assert (out == 7.0).all()  # nothing outside the view was written


def test_rotary_inverse_and_gradient():
    """inverse undoes a rotation; the gradient of <c, rotary(x)> is the inverse rotation of c, by differences in 64 bits."""
    g = gen(3)
    pos = torch.randint(0, 5000, (5,), generator=g, device="cuda", dtype=torch.int32)
    f = ops.rotary_frequencies(32)
    x, c = randn(g, 5, 3, 48), randn(g, 5, 3, 48)
    y = ops.rotary(x, pos, f, offset=8)
    assert torch.allclose(ops.rotary(y, pos, f, offset=8, inverse=True), x, atol=3e-6)
    grad = ops.rotary(c, pos, f, offset=8, amplitude=1.3, inverse=True)
    full = lambda v: torch.cat((v[..., :8], turned(v[..., 8:40], pos, f, "interleaved", 1.3), v[..., 40:].double()), -1)
    for at in ((0, 0, 8), (2, 1, 39), (4, 2, 20), (1, 1, 3)):
        d = torch.zeros_like(x, dtype=torch.float64)
        d[at] = 1e-3
        slope = ((full(x.double() + d) - full(x.double() - d)) * c.double()).sum() / 2e-3
        assert abs(float(slope) - float(grad[at])) < 1e-5
    with pytest.raises(ValueError, match="forward only"):
        ops.rotary(x.requires_grad_(), pos, f)


def test_rotary_empty():
    f = ops.rotary_frequencies(32)
    assert ops.rotary(torch.zeros(0, 4, 64, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), f).shape == (0, 4, 64)
    assert ops.rotary(torch.zeros(3, 0, 64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), f).shape == (3, 0, 64)


# ------------------------------------------------------------- append -----
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("tokens,rank,rot,block,blocks", [(1, 512, 64, 16, 4), (64, 512, 64, 16, 40), (37, 128, 32, 12, 5), (1000, 256, 64, 1, 1300),
                                                          (5, 100, 6, 3, 7), (3, 1, 2, 64, 1), (129, 77, 256, 7, 20)])
def test_append(tokens, rank, rot, block, blocks, dtype, layout):
    g = gen(tokens + rank)
    latent, key = randn(g, tokens, rank, dtype=dtype), randn(g, tokens, rot, dtype=dtype)
    pos = torch.randint(0, 200000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    slots = torch.randperm(blocks * block, generator=g, device="cuda")[:tokens].contiguous()
    slots[::5] = -1
    if tokens > 3:
        slots[1], slots[2] = blocks * block, 2 ** 40  # past the end: nothing is written
    f = ops.rotary_frequencies(rot)
    cache = randn(g, blocks, block, rank + rot, dtype=dtype)
    before = cache.clone()
    assert ops.latent_append(latent, key, pos, f, slots, cache, layout=layout, amplitude=1.1) is cache
    kept = (slots >= 0) & (slots < blocks * block)
    rows = cache.view(-1, rank + rot)
    assert torch.equal(rows[slots[kept], :rank], latent[kept])
    if kept.any():
        check_rotary(key[kept][:, None], pos[kept], f, rows[slots[kept], rank:][:, None], layout, 0, 1.1)
    other = torch.ones(blocks * block, dtype=torch.bool, device="cuda")
    other[slots[kept]] = False
    assert torch.equal(rows[other], before.view(-1, rank + rot)[other])


def test_append_strides():
    """A cache that is one layer of several, rows with a gap, inputs that are slices of one projection."""
    g = gen(5)
    both = randn(g, 40, 3 + 512 + 64, dtype=BF)
    latent, key = both[:, 3:515], both[:, 515:]
    store = torch.zeros(9, 2, 16, 600, device="cuda", dtype=BF)
    cache = store[:, 1, :, 5:581]
    slots = torch.randperm(144, generator=g, device="cuda")[:40].contiguous()
    pos = torch.arange(40, device="cuda")
    f = ops.rotary_frequencies(64)
    ops.latent_append(latent, key, pos, f, slots, cache, layout="half")
    got = cache[slots // 16, slots % 16]
    assert torch.equal(got[:, :512], latent)
    check_rotary(key[:, None], pos, f, got[:, 512:][:, None], "half", 0)
    cache.zero_()
    assert not store.any()


# ------------------------------------------------------------- decode -----
def decode_case(lengths, new, heads, rank, key_dim, block, dtype, seed=0, spare=2, junk=float("nan")):
    g = gen(seed)
    need = [-(-max(n, 0) // block) for n in lengths]
    blocks = sum(need) + spare
    order = torch.randperm(blocks, generator=g, device="cuda").int()
    table = torch.full((len(lengths), max(need + [1]) + 1), -7, dtype=torch.int32, device="cuda")
    cache = torch.full((blocks, block, rank + key_dim), junk, device="cuda", dtype=dtype)
    at = 0
    for b, n in enumerate(lengths):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        rows = randn(g, n, rank + key_dim, dtype=dtype)
        for i in range(need[b]):
            part = rows[i * block:(i + 1) * block]
            cache[int(table[b, i]), :len(part)] = part
    q = randn(g, len(lengths), new, heads, rank + key_dim, dtype=dtype)
    return q, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda")


def check_decode(q, cache, table, lengths, rank, scale, out, lse):
    _, new, heads, width = q.shape
    u = U[q.dtype]
    for b, n in enumerate(lengths.tolist()):
        n = min(n, table.shape[1] * cache.shape[1])
        ids = table[b, :-(-n // cache.shape[1]) if n > 0 else 0].long()
        rows = torch.cat([cache[i] if 0 <= i < cache.shape[0] else torch.zeros_like(cache[0]) for i in ids.tolist()] or [cache[0][:0]])[:max(n, 0)].double()
        for t in range(new):
            sees = n - new + 1 + t
            if sees <= 0:
                assert not out[b, t].any() and (lse[b, t] == -math.inf).all()
                continue
            s = q[b, t].double() @ rows[:sees].T * scale
            p = torch.softmax(s, 1)
            want, mag = p @ rows[:sees, :rank], p @ rows[:sees, :rank].abs()
            off = (out[b, t].double() - want).abs()
            assert (off <= u * want.abs() + (2 * u + 1e-5) * mag + 1e-7).all(), (b, t, float((off / mag).max()))
            assert torch.allclose(lse[b, t].double(), torch.logsumexp(s, 1), rtol=1e-6, atol=1e-5), (b, t)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lengths,new,heads,rank,key_dim,block", [
    ([1], 1, 1, 512, 64, 16), ([0], 1, 16, 512, 64, 16), ([0, 5, 0, 1], 1, 16, 512, 64, 16), ([63, 64, 65, 127, 128, 129], 1, 16, 512, 64, 16),
    ([777], 1, 16, 512, 64, 16), ([300, 2, 1000], 1, 128, 512, 64, 16), ([200, 31], 1, 65, 512, 64, 12), ([500], 1, 64, 256, 32, 7),
    ([90, 400], 3, 16, 512, 64, 64), ([2, 5, 1], 5, 3, 512, 64, 16), ([64, 65, 66], 4, 17, 128, 64, 1), ([333], 1, 130, 512, 0, 16),
    ([1025, 17], 2, 40, 64, 8, 48), ([3000], 1, 20, 512, 64, 16), ([40] * 70, 1, 5, 192, 40, 16), ([4100, 1, 0, 2500, 64], 7, 10, 512, 64, 33),
    ([k * 7 % 90 for k in range(300)], 1, 4, 128, 64, 16), ([700, 130], 2, 96, 512, 64, 32), ([500, 0, 77], 4, 64, 256, 64, 24)])
def test_decode(lengths, new, heads, rank, key_dim, block, dtype):
    q, cache, table, n = decode_case(lengths, new, heads, rank, key_dim, block, dtype, seed=len(lengths) + heads)
    scale = 1.7 / math.sqrt(rank + key_dim)
    out = torch.full((len(lengths), new, heads, rank), float("nan"), device="cuda", dtype=dtype)
    got, lse = ops.latent_decode(q, cache, table, n, scale=scale, out=out)
    assert got is out
    check_decode(q, cache, table, n, rank, scale, out, lse)
    again, lse2 = ops.latent_decode(q, cache, table, n, scale=scale, out=torch.empty_like(out))
    assert torch.equal(again, out) and torch.equal(lse2, lse)  # the same bits


@pytest.mark.parametrize("dtype", [BF, HF])
def test_decode_peaked_and_negative_scores(dtype):
    """One row far above the others, then all scores far below zero, then growing along the cache (the running maximum moves at every tile)."""
    q, cache, table, n = decode_case([700, 700, 700], 1, 16, 512, 64, 16, dtype, seed=9)
    cache[int(table[0, 20]), 3] *= 6
    rows = table[2, :44].long()
    up = torch.linspace(0, 3, 704, device="cuda").reshape(44, 16, 1).to(dtype)
    cache[rows] = torch.nan_to_num(cache[rows]) * up + q[2, 0, 0] * up * 0.1
    for scale in (0.3, -0.2, 0.0):
        out, lse = ops.latent_decode(q, cache, table, n, scale=scale)
        check_decode(q, cache, table, n, 512, scale, out, lse)


def test_decode_table_and_lengths_out_of_range():
    """Entries outside the cache stand for zeros, a length past the table for the table's end; neither reaches other memory."""
    q, cache, table, n = decode_case([100, 90], 1, 16, 512, 64, 16, BF, seed=4, junk=0.5)
    table[0, 2], table[1, 1] = cache.shape[0], 2 ** 31 - 1
    table[0, 7:] = -1
    n[0] = 2 ** 31 - 1
    out, lse = ops.latent_decode(q, cache, table, n, scale=0.05)
    check_decode(q, cache, table, n, 512, 0.05, out, lse)
    n[0] = -5
    out, lse = ops.latent_decode(q, cache, table, n, scale=0.05)
    assert not out[0].any() and (lse[0] == -math.inf).all()


@pytest.mark.parametrize("lengths", [[60, 40], [5000, 40]])  # whole requests, and joined parts
@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
def test_decode_numbers_that_are_none_show(lengths, junk):
    """A score that is NaN or +infinity makes the row's result NaN, not zero; other requests keep theirs."""
    q, cache, table, n = decode_case(lengths, 1, 16, 512, 64, 16, BF, seed=13)
    want, lse = ops.latent_decode(q, cache, table, n, scale=0.05)
    q[0, 0, 3, 100] = 1.0
    cache[int(table[0, 1]), 5, 100] = junk
    out, lse2 = ops.latent_decode(q, cache, table, n, scale=0.05)
    assert out[0, 0, 3].isnan().all() and lse2[0, 0, 3].isnan()
    assert torch.equal(out[1], want[1]) and torch.equal(lse2[1], lse[1])


def test_decode_strides():
    g = gen(6)
    q, cache, table, n = decode_case([150, 40], 2, 6, 512, 64, 16, BF, seed=6)
    wide = torch.zeros(2, 2, 3, 6, 600, device="cuda", dtype=BF)
    qv = wide[:, :, 1, :, 8:584]
    qv.copy_(q)
    store = torch.full((cache.shape[0], 3, 16, 584), float("nan"), device="cuda", dtype=BF)
    cv = store[:, 2, :, :576]
    cv.copy_(cache)
    tv = torch.zeros(2, 40, dtype=torch.int32, device="cuda")[:, 3:3 + table.shape[1]]
    tv.copy_(table)
    ov = torch.zeros(2, 6, 2, 520, device="cuda", dtype=BF).transpose(1, 2)[..., 8:]
    a, la = ops.latent_decode(q, cache, table, n, scale=0.05)
    b, lb = ops.latent_decode(qv, cv, tv, n, scale=0.05, out=ov)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_decode_offsets_past_32_bits():
    """A cache of more than 2^32 bytes and 2^31 elements: rows at its far end."""
    blocks = 240000
    cache = torch.zeros(blocks, 16, 576, device="cuda", dtype=BF)
    g = gen(7)
    ids = [blocks - 1, 0, blocks - 2, 233100, 117000]
    for i in ids:
        cache[i] = randn(g, 16, 576, dtype=BF)
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    q = randn(g, 1, 1, 16, 576, dtype=BF)
    n = torch.tensor([77], dtype=torch.int32, device="cuda")
    out, lse = ops.latent_decode(q, cache, table, n, scale=0.06)
    check_decode(q, cache, table, n, 512, 0.06, out, lse)
    slots = torch.tensor([(blocks - 1) * 16 + 3], device="cuda")
    lat, key = randn(g, 1, 512, dtype=BF), randn(g, 1, 64, dtype=BF)
    ops.latent_append(lat, key, torch.zeros(1, dtype=torch.int32, device="cuda"), ops.rotary_frequencies(64), slots, cache)
    assert torch.equal(cache[-1, 3], torch.cat((lat, key), 1)[0])


def test_decode_on_another_stream():
    q, cache, table, n = decode_case([600, 1200], 1, 32, 512, 64, 16, BF, seed=8)
    want = ops.latent_decode(q, cache, table, n, scale=0.05)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    late = torch.zeros_like(q)
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        late.copy_(q)  # the kernel must come after this copy, on s
        got = ops.latent_decode(late, cache, table, n, scale=0.05)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_calls_in_a_row_keep_their_order():
    """Kernels whose blocks are set up early still see all that earlier calls wrote: the same bits as with a wait after every call."""
    def steps(wait):
        g = gen(31)
        q, cache, table, n = decode_case([900, 70, 300], 1, 16, 512, 64, 16, BF, seed=31, junk=0.0)
        x, pos = randn(g, 3000, 4, 64, dtype=BF), torch.arange(3000, device="cuda")
        latent, key, at = randn(g, 3, 512, dtype=BF), randn(g, 3, 64, dtype=BF), torch.tensor([5, 9, 2], device="cuda")
        f, u = ops.rotary_frequencies(64), torch.full((3,), 0.37, device="cuda")
        rows = torch.arange(3, device="cuda")
        prompt = prefill_case([200, 90], [700, 90], 2, 64, 64, 64, BF, seed=31)
        tokens, outs = [], [torch.empty(3, 1, 16, 512, device="cuda", dtype=BF) for _ in range(2)] + [torch.empty(290, 2, 64, device="cuda", dtype=BF)]
        for i in range(25):
            slot = table[rows, 2].long() * 16 + i % 16  # a row of the third block, seen by every request
            for call in (lambda: ops.rotary(x, pos, f, layout="half", out=x), lambda: ops.rotary(x, pos, f, layout="half", inverse=i % 3 == 0, out=x),
                         lambda: ops.rotary(q[:, 0, :, 512:], at, f, out=q[:, 0, :, 512:]),
                         lambda: ops.latent_append(latent, key, at, f, slot, cache),
                         lambda: ops.latent_decode(q, cache, table, n, scale=0.1, out=outs[0]),
                         lambda: ops.latent_decode(q, cache, table, n, scale=0.3, out=outs[1]),
                         lambda: ops.rotary(outs[0][:, 0], at, f, out=outs[0][:, 0]), lambda: q[..., :512].copy_(outs[0] + outs[1]),
                         lambda: ops.rotary(prompt[0], at.new_zeros(290) + i, f, layout="half", offset=64, out=prompt[0]),
                         lambda: ops.latent_prefill(*prompt, scale=0.2, longest=200, out=outs[2]), lambda: prompt[0][..., :64].copy_(outs[2]),
                         lambda: tokens.append(ops.sample(q[:, 0].reshape(3, -1), u, top_k=rows.int() + 5)[0])):
                call()
                if wait:
                    torch.cuda.synchronize()
        return [x, q, cache, prompt[0], torch.stack(tokens)]
    want = steps(True)
    assert all(torch.equal(a, b) for _ in range(3) for a, b in zip(steps(False), want))


def test_operators_in_a_graph():
    q, cache, table, n = decode_case([600, 1200], 1, 32, 512, 64, 16, BF, seed=8)
    logits, u = torch.randn(2, 5000, device="cuda", generator=gen(1)), torch.tensor([0.3, 0.8], device="cuda")
    call = lambda: (*ops.latent_decode(q, cache, table, n, scale=0.05), *ops.sample(logits, u))
    want = [t.clone() for t in call()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    q.mul_(2)
    n[0] = 300
    logits.mul_(0.5)
    want = [t.clone() for t in call()]
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------ prefill -----
def prefill_case(nq, nk, heads, head, rot, value, dtype, seed=0):
    g = gen(seed)
    offs = [torch.tensor(np.cumsum([0] + list(n)), dtype=torch.int32, device="cuda") for n in (nq, nk)]
    return (randn(g, sum(nq), heads, head + rot, dtype=dtype), randn(g, sum(nk), heads, head, dtype=dtype),
            randn(g, sum(nk), rot, dtype=dtype), randn(g, sum(nk), heads, value, dtype=dtype), *offs)


def check_prefill(q, key, shared, value, q_offsets, k_offsets, scale, out, lse, causal=True):
    u = U[q.dtype]
    qo, ko = q_offsets.tolist(), k_offsets.tolist()
    for a, b, c, d in zip(qo, qo[1:], ko, ko[1:]):
        if b == a:
            continue
        hidden = torch.ones(b - a, d - c, dtype=torch.bool, device="cuda").triu(d - c - (b - a) + 1)
        for h in range(q.shape[1]):
            k = torch.cat((key[c:d, h], shared[c:d]), 1).double()
            s = q[a:b, h].double() @ k.T * scale
            if causal:
                s = s.masked_fill(hidden, -math.inf)
            some = torch.isfinite(s).any(1)
            assert not out[a:b, h][~some].any() and (lse[a:b, h][~some] == -math.inf).all()
            if not some.any():
                continue
            p = torch.softmax(s[some], 1)
            v = value[c:d, h].double()
            want, mag = p @ v, p @ v.abs()
            off = (out[a:b, h][some].double() - want).abs()
            assert (off <= u * want.abs() + (2 * u + 1e-5) * mag + 1e-7).all(), (a, h, float((off / mag).max()))
            assert torch.allclose(lse[a:b, h][some].double(), torch.logsumexp(s[some], 1), rtol=1e-6, atol=1e-5)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("nq,nk,heads,head,rot,value", [
    ([1], [1], 1, 128, 64, 128), ([1, 1, 1], [1, 2, 300], 2, 128, 64, 128), ([127, 128, 129], [127, 128, 129], 2, 128, 64, 128),
    ([255, 0, 257, 1], [255, 0, 257, 1], 1, 128, 64, 128), ([64, 10], [500, 10], 3, 128, 64, 128), ([300], [300], 4, 64, 32, 64),
    ([50, 3, 77], [20, 3, 76], 2, 128, 64, 128), ([40, 5], [0, 5], 1, 128, 64, 128), ([33], [99], 5, 8, 8, 8), ([130], [700], 1, 72, 40, 104),
    ([20], [150], 2, 128, 0, 128), ([1000], [1000], 1, 128, 64, 128), ([513], [2049], 2, 64, 64, 128),
    ([k * 37 % 301 for k in range(40)], [k * 37 % 301 + k % 3 * 50 for k in range(40)], 12, 64, 64, 64),
    ([600, 0, 3, 270] * 3, [1, 200, 900, 270] * 3, 40, 128, 64, 128), ([40] * 150, [40] * 150, 5, 16, 8, 24)])
def test_prefill(nq, nk, heads, head, rot, value, dtype, causal):
    args = prefill_case(nq, nk, heads, head, rot, value, dtype, seed=sum(nq))
    scale = 1.7 / math.sqrt(head + rot)
    out = torch.full((sum(nq), heads, value), float("nan"), device="cuda", dtype=dtype)
    got, lse = ops.latent_prefill(*args, scale=scale, longest=max(nq), causal=causal, out=out)
    assert got is out
    check_prefill(*args, scale, out, lse, causal)
    again, lse2 = ops.latent_prefill(*args, scale=scale, longest=max(nq), causal=causal)
    assert torch.equal(again, out) and torch.equal(lse2, lse)  # the same bits
    check_prefill(*args, scale, *ops.latent_prefill(*args, scale=scale, longest=max(nq) + 1000, causal=causal), causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("nq,nk,heads,head,rot,value", [
    ([1], [9000], 1, 128, 64, 128), ([300, 1, 17, 256], [5000, 2000, 40, 256], 1, 128, 64, 128), ([4000], [4000], 1, 64, 64, 64),
    ([513, 513], [1300, 3001], 3, 72, 40, 104), ([700, 0], [600, 5000], 2, 128, 64, 8), ([257], [8192], 8, 128, 0, 128)])
def test_prefill_keys_shared_by_blocks(nq, nk, heads, head, rot, value, dtype, causal):
    """Few queries and many keys, where blocks take stretches of the keys and join their sums."""
    args = prefill_case(nq, nk, heads, head, rot, value, dtype, seed=sum(nk))
    args[1][nk[0] // 3] *= 6  # one block's maximum far above the others'
    scale = 1.7 / math.sqrt(head + rot)
    out = torch.full((sum(nq), heads, value), float("nan"), device="cuda", dtype=dtype)
    lse = torch.full((sum(nq), heads), float("nan"), device="cuda")
    ops.latent_prefill(*args, scale=scale, longest=max(nq), causal=causal, out=out, lse=lse)
    check_prefill(*args, scale, out, lse, causal)
    again, lse2 = ops.latent_prefill(*args, scale=scale, longest=max(nq), causal=causal)
    assert torch.equal(again, out) and torch.equal(lse2, lse)  # the same bits


def test_prefill_requests_do_not_reach_each_other():
    """NaN and infinities in one request's keys and values, and in rows past the last offset, leave the others' rows untouched."""
    nq = nk = [70, 33, 150]
    q, key, shared, value, qo, ko = prefill_case(nq, nk, 2, 128, 64, 128, BF, seed=3)
    more = [torch.cat((t, torch.full_like(t[:60], float("nan")))) for t in (q, key, shared, value)]
    want, lse = ops.latent_prefill(*more, qo, ko, scale=0.1, longest=150)
    check_prefill(q, key, shared, value, qo, ko, 0.1, want[:253], lse)
    for t, junk in ((1, float("nan")), (2, float("inf")), (3, float("nan")), (3, float("-inf"))):
        bad = [x.clone() for x in more]
        bad[t][70:103] = junk
        out, lse2 = ops.latent_prefill(*bad, qo, ko, scale=0.1, longest=150)
        keep = [*range(70), *range(103, 253)]
        assert torch.equal(out[keep], want[keep]) and torch.equal(lse2[keep], lse[keep])


def test_prefill_later_keys_do_not_count():
    """Causal: NaN in keys after a query's own leave it untouched, to the row."""
    args = prefill_case([200], [200], 2, 128, 64, 128, HF, seed=2)
    want, lse = ops.latent_prefill(*args, scale=0.1, longest=200)
    args[1][150:] = float("nan")
    out, lse2 = ops.latent_prefill(*args, scale=0.1, longest=200)
    assert torch.equal(out[:150], want[:150]) and torch.equal(lse2[:150], lse[:150])


@pytest.mark.parametrize("nk", [200, 3000])
@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
def test_prefill_numbers_that_are_none_show(nk, junk):
    args = prefill_case([200], [nk], 2, 128, 64, 128, BF, seed=2)
    want, lse = ops.latent_prefill(*args, scale=0.1, longest=200)
    args[0][:, 1, 7] = 1.0
    args[1][nk - 50, 1, 7] = junk
    out, lse2 = ops.latent_prefill(*args, scale=0.1, longest=200)
    assert out[150:, 1].isnan().all() and lse2[150:, 1].isnan().all()
    assert torch.isfinite(out[:150, 1]).all() and torch.equal(out[:, 0], want[:, 0]) and torch.equal(lse2[:, 0], lse[:, 0])


def test_prefill_strides_and_bounds():
    nq, nk = [90, 60], [140, 60]
    q, key, shared, value, qo, ko = prefill_case(nq, nk, 3, 128, 64, 128, BF, seed=5)
    want, lse = ops.latent_prefill(q, key, shared, value, qo, ko, scale=0.1, longest=90)
    kv = torch.zeros(200, 3, 264, device="cuda", dtype=BF)  # keys and values of one projection
    kv[..., :128], kv[..., 136:] = key, value
    qt = q.transpose(0, 1).contiguous().transpose(0, 1)
    st = torch.zeros(200, 80, device="cuda", dtype=BF)
    st[:, 16:] = shared
    ot = torch.zeros(150, 3, 256, device="cuda", dtype=BF)
    out, lse2 = ops.latent_prefill(qt, kv[..., :128], st[:, 16:], kv[..., 136:], qo, ko, scale=0.1, longest=90, out=ot[..., 64:192])
    assert torch.equal(out, want) and torch.equal(lse2, lse)
    assert not ot[..., :64].any() and not ot[..., 192:].any()
    # fewer queries computed than there are: the rest is not written
    out = torch.full_like(want, 7.0)
    ops.latent_prefill(q, key, shared, value, qo, ko, scale=0.1, longest=70, out=out)
    assert torch.equal(out[:70], want[:70]) and (out[70:90] == 7.0).all() and torch.equal(out[90:], want[90:])
    # offsets past the rows are bounded by them
    qo[2], ko[2] = 2 ** 31 - 1, 2 ** 31 - 1
    out, lse2 = ops.latent_prefill(q, key, shared, value, qo, ko, scale=0.1, longest=200)
    assert torch.equal(out, want) and torch.equal(lse2, lse)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_prefill_moving_maximum(dtype):
    """Scores that grow along the keys, and rows far apart in size: the running maximum moves at every tile."""
    q, key, shared, value, qo, ko = prefill_case([300], [900], 2, 128, 64, 128, dtype, seed=6)
    up = torch.linspace(0, 4, 900, device="cuda")[:, None]
    shared = (shared + up * q[0, 0, 128:].float() * 0.2).to(dtype)
    q[:, :, 128:] = q[0, 0, 128:]
    for scale in (0.5, -0.4, 0.0):
        out, lse = ops.latent_prefill(q, key, shared, value, qo, ko, scale=scale, longest=300)
        check_prefill(q, key, shared, value, qo, ko, scale, out, lse)


def test_forms_agree():
    """The absorbed form over a cache and the expanded form over its expansion are the same attention."""
    g = gen(11)
    n, heads = 190, 4
    latent, shared = randn(g, n, 512, dtype=BF), randn(g, n, 64, dtype=BF)
    up = randn(g, heads, 512, 128) / 24
    key = torch.einsum("nr,hrd->nhd", latent.float(), up)
    q = randn(g, 1, heads, 192)
    absorbed = torch.cat((torch.einsum("hd,hrd->hr", q[0, :, :128], up), q[0, :, 128:]), 1)
    _, lse_e = ops.latent_prefill(q.to(BF), key.to(BF), shared, key.to(BF), torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
                                  torch.tensor([0, n], dtype=torch.int32, device="cuda"), scale=0.07, longest=1)
    cache = torch.zeros(12, 16, 576, device="cuda", dtype=BF)
    cache.view(-1, 576)[:n] = torch.cat((latent, shared), 1)
    out, lse_a = ops.latent_decode(absorbed.to(BF)[None, None], cache, torch.arange(12, dtype=torch.int32, device="cuda")[None],
                                   torch.tensor([n], dtype=torch.int32, device="cuda"), scale=0.07)
    assert torch.allclose(lse_a.flatten(), lse_e.flatten(), atol=0.03)  # both sides round their operands to bfloat16


# ------------------------------------------------------------- sample -----
EDGE = 3e-6  # weights are 32-bit exponentials: a cut or a draw this near an edge (as a share of the weight) may go either way


def sampled(row, u, t=1.0, k=0, p=1.0, m=0.0):
    """The definition in 64 bits, as {token: logprob}: one token, or one more for each edge that is too near to call."""
    row = np.where(np.isnan(row), -np.inf, row.astype(np.float64))
    top = row.max()
    if top == -np.inf:
        return {-1: -math.inf}
    if not t > 0:
        return {int(np.argmax(row)): 0.0}
    w = (row == np.inf).astype(float) if top == np.inf else np.exp((row - top) / t)
    order = np.argsort(-row, kind="stable")
    if 0 < k < len(row):
        order = order[:k]
    mass = np.cumsum(w[order])
    before = mass - w[order]
    some = {}
    for edge in (0.0, -EDGE, EDGE) if p < 1 else (0.0,):
        nucleus = order[(before < (p + edge) * mass[-1]) | (np.arange(len(order)) == 0)] if p < 1 else order
        kept = np.sort(nucleus[w[nucleus] >= min(m, 1.0)])
        sums = np.cumsum(w[kept])
        for du in (0.0, -EDGE, EDGE):
            at = min(int(np.searchsorted(sums, (u + du) * sums[-1], side="right")), len(kept) - 1)
            some.setdefault(int(kept[at]), math.log(w[kept[at]] / sums[-1]) if w[kept[at]] > 0 else -math.inf)
    return some


def check_sample(logits, u, got, **par):
    token, logprob = (x.cpu().numpy() for x in got)
    x, uu = logits.float().cpu().numpy(), u.cpu().numpy().astype(np.float64)
    par = {k: v.cpu().numpy().astype(np.float64) if k != "k" else v.cpu().numpy() for k, v in par.items() if v is not None}
    for b in range(len(x)):
        some = sampled(x[b], uu[b], **{k: v[b] for k, v in par.items()})
        assert int(token[b]) in some, (b, token[b], some)
        lp = some[int(token[b])]
        assert (lp == logprob[b]) or abs(lp - logprob[b]) < 5e-6 * max(1, abs(lp)), (b, lp, logprob[b])


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (5, 31), (4, 33), (9, 1000), (3, 1025), (2, 4099), (7, 32000), (2, 100003), (300, 257), (1, 300000)])
def test_sample(rows, vocab, dtype):
    g = gen(vocab)
    logits = (randn(g, rows, vocab) * 3).to(dtype)
    u = torch.rand(rows, generator=g, device="cuda")
    pick = lambda *v: torch.tensor(v, device="cuda")[torch.randint(0, len(v), (rows,), generator=g, device="cuda")]
    check_sample(logits, u, ops.sample(logits, u))
    for _ in range(4):
        t, k, p, m = pick(0.3, 0.8, 1.0, 2.5), pick(0, 1, 2, 20, 900, 10 ** 6).int(), pick(1.0, 0.95, 0.7, 0.1), pick(0.0, 0.0, 0.02, 0.3)
        check_sample(logits, u, ops.sample(logits, u, temperature=t, top_k=k, top_p=p, min_p=m), t=t, k=k, p=p, m=m)
        check_sample(logits, u, ops.sample(logits, u, top_p=p), p=p)
        check_sample(logits, u, ops.sample(logits, u, top_k=k, temperature=t), k=k, t=t)


@pytest.mark.parametrize("vocab", [5, 700, 40000])
def test_sample_ties(vocab):
    """Few distinct values: the cut lies inside a group of equals and the lowest indices stay."""
    g = gen(vocab)
    rows = 24
    logits = torch.randint(0, 3, (rows, vocab), generator=g, device="cuda").to(BF)
    logits[0] = 1.5
    logits[1] = 0.0
    logits[1, ::2] = -0.0
    u = torch.rand(rows, generator=g, device="cuda")
    k = torch.randint(1, vocab + 1, (rows,), generator=g, device="cuda").int()
    p = torch.rand(rows, generator=g, device="cuda") * 0.9 + 0.05
    check_sample(logits, u, ops.sample(logits, u, top_k=k), k=k)
    check_sample(logits, u, ops.sample(logits, u, top_p=p), p=p)
    check_sample(logits, u, ops.sample(logits, u, top_k=k, top_p=p), k=k, p=p)
    half = torch.full((rows,), 0.5, device="cuda")
    for last in (0.0, 1 - 2.0 ** -24):
        ends = torch.full((rows,), last, device="cuda")
        token, _ = ops.sample(logits[:2], ends[:2], top_k=k[:2])
        assert token.tolist() == [0, 0] if last == 0 else token.tolist() == (k[:2] - 1).tolist()
    token, lp = ops.sample(logits[:1].float(), ends[:1], top_p=half[:1])
    assert int(token) == -(-vocab // 2) - 1 and abs(float(lp) + math.log(-(-vocab // 2))) < 1e-5


def test_sample_special_values():
    nan, inf = float("nan"), float("inf")
    rows = [[-inf] * 6, [nan] * 6, [nan, 1, -inf, 1, nan, 0], [inf, 0, inf, nan, -inf, 3], [-inf, -inf, 2, -inf, -inf, -inf],
            [-3e38, -3e38, -3.4e38, -inf, -3e38, nan], [3e38, -3e38, 0, 0, 0, 0], [0, 0, 0, 0, 0, 0]]
    x = torch.tensor(rows, device="cuda")
    u = torch.full((8,), 0.6, device="cuda")
    token, lp = ops.sample(x, u)
    assert token.tolist() == [-1, -1, 3, 2, 2, 1, 0, 3]
    assert lp[:2].tolist() == [-inf, -inf]
    z = math.log(2 + math.exp(-1))
    assert torch.allclose(lp[2:].cpu(), torch.tensor([-z, -math.log(2), 0, -math.log(3), 0, -math.log(6)]), atol=1e-6)
    vec = lambda v, d=F32: torch.full((8,), v, device="cuda", dtype=d)
    for greedy in (0.0, -1.0, nan):
        token, lp = ops.sample(x, u, temperature=vec(greedy), top_k=vec(3, torch.int32), min_p=vec(0.5))
        assert token.tolist() == [-1, -1, 1, 0, 2, 0, 0, 0] and lp[2:].tolist() == [0.0] * 6
    for par in (dict(top_p=vec(0.0)), dict(top_p=vec(-1.0)), dict(top_k=vec(1, torch.int32))):
        token, lp = ops.sample(x, u, **par)
        assert token.tolist() == [-1, -1, 1, 0, 2, 0, 0, 0], par
    token, _ = ops.sample(x, u, min_p=vec(2.0))  # above one: the largest, and its equals
    assert token.tolist() == [-1, -1, 3, 2, 2, 1, 0, 3]
    token, _ = ops.sample(x, vec(nan), min_p=vec(nan), top_p=vec(nan))
    assert token.tolist() == [-1, -1, 1, 0, 2, 0, 0, 0]
    token, _ = ops.sample(x, vec(1.0))
    assert token.tolist() == [-1, -1, 5, 2, 2, 4, 0, 5]
    token, _ = ops.sample(x, vec(0.6), temperature=vec(1e-30))
    assert token.tolist()[2:5] == [3, 2, 2]


def test_sample_strides_and_frequencies():
    """Rows with a gap; and the draws follow the distribution (chi-squared at 40,000 draws, 9 kept tokens)."""
    g = gen(12)
    base = randn(g, 6, 513)
    u = torch.rand(6, generator=g, device="cuda")
    for first in (0, 1, 3):
        x = base[:, first:first + 500]
        a = ops.sample(x, u)
        b = ops.sample(x.contiguous(), u)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    n = 40000
    x = torch.tensor([2.0, 0.5, -1.0, 1.2, 0.0, 0.3, -0.2, 1.9, -5.0, 0.1], device="cuda").repeat(n, 1)
    k = torch.full((n,), 9, dtype=torch.int32, device="cuda")
    token, _ = ops.sample(x, torch.rand(n, generator=g, device="cuda"), top_k=k)
    p = torch.softmax(torch.where(x[0] > -4, x[0].double(), -math.inf), 0)
    count = torch.bincount(token, minlength=10).double()
    kept = p > 0
    assert count[~kept].sum() == 0
    assert float(((count - n * p)[kept] ** 2 / (n * p)[kept]).sum()) < 30  # 8 degrees of freedom: P(> 30) is 2e-4
