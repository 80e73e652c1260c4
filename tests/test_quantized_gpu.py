"""The 8-bit block cache on the GPU: rows that are appended and attention over
them against their formulas in 64 bits, at the sizes and values where they can go wrong.

Tolerances, from the arithmetic.  A number stored in 8 bits (four significant bits, multiples of 2^-9) is off by at
most half its step, 2^-4 of itself or 2^-10, and a rotated key by what 32 bits leave
(2e-6 of the pair's length, which may also tip a rounding); latents are rounded once and
compared exactly.  An attention's result of unit roundoff u / 2 (bfloat16: u = 2^-8) is off by u / 2 |y| for its own rounding, u / 2 sum_j p_j |v_j|
for the weights' (a weight is rounded by 1.25 * 2^-9 or 1.5 * 2^-11 of itself); twice that is allowed, and 1e-5 of the same sum for 32-bit
arithmetic.  A query's elements may be off by 2^-21 of its largest, so that a
score is by 2^-21 max |q| sum |c| |scale|, its weight by twice that, and lse by as much."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_ops_gpu import turned  # noqa: E402

pytestmark = pytest.mark.gpu

BF, HF, F32, E4 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
U = {BF: 2.0 ** -8, HF: 2.0 ** -11}


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


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def bits(t):
    return t.view(torch.uint8)


def half_step(x):
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -6))) - 4)


def nearest(x):
    """x (64-bit) in 8 bits, the numbers they stand for: ties to even, 448 at most, infinities as NaN."""
    step = 2 * half_step(x)
    y = (torch.round(x / step) * step).clamp(-448, 448)
    return torch.where(torch.isfinite(x), y, torch.full_like(y, math.nan))


def scale_for(x):
    """The smallest power of two in [2^-60, 2^60] with |x| <= 448 times it, of the finite ones."""
    a = float(torch.where(torch.isfinite(x), x, torch.zeros_like(x)).abs().max())
    e = -60
    while e < 60 and a > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


# ------------------------------------------------------------- append -----
def placed(lengths, block, seed, spare=3, width=0):
    """A table that puts requests of these lengths into blocks anywhere, and the number of blocks."""
    need = [-(-max(n, 0) // block) for n in lengths]
    order = np.random.RandomState(seed).permutation(sum(need) + spare)
    table, at = torch.full((len(lengths), max(max(need + [1]), width)), -9, dtype=torch.int32), 0
    for b, k in enumerate(need):
        table[b, :k] = torch.from_numpy(order[at:at + k].astype(np.int32))
        at += k
    return table.cuda(), sum(need) + spare


def check_append(latent, key, f, offsets, table, lengths, before, after, layout, amplitude=1.0):
    """Both states are (cache, scales); everything that is not to change must have its bits."""
    (cache, scales), (got, got_scales) = before, after
    blocks, block, width = cache.shape
    rank, o, L = latent.shape[1], offsets.tolist(), lengths.tolist()
    same = torch.ones(blocks, block, dtype=torch.bool, device="cuda")
    for b in range(len(L)):
        lo, hi = (min(max(v, 0), latent.shape[0]) for v in o[b:b + 2])
        tokens = [(p, hi - L[b] + p) for p in range(max(L[b] - (hi - lo), 0), min(L[b], table.shape[1] * block))]
        for blk in sorted({p // block for p, _ in tokens}):
            i = int(table[b, blk])
            if not 0 <= i < blocks:
                continue
            here = [(p % block, n) for p, n in tokens if p // block == blk]
            rows, source = [r for r, _ in here], [n for _, n in here]
            pos = torch.tensor([blk * block + r for r in rows])
            parts = (latent[source].double(), turned(key[source][:, None], pos, f, layout, amplitude)[:, 0])
            same[i, rows] = False
            for part, cols, x in ((0, slice(0, rank), parts[0]), (1, slice(rank, width), parts[1])):
                scale, had = scale_for(x), float(scales[i, part])
                if rows[0]:
                    scale = min(max(had, scale), 2.0 ** 60)
                assert float(got_scales[i, part]) == scale, (b, blk, part)
                y = got[i, rows][:, cols].double()
                if part == 0:
                    assert torch.equal(torch.nan_to_num(y, 999.0), torch.nan_to_num(nearest(x / scale), 999.0)), (b, blk)
                else:
                    fine = torch.isfinite(x)
                    assert torch.equal(torch.isnan(y), ~fine)
                    tip = 2e-6 * abs(amplitude) * key[source].double().nan_to_num(0.0, 0.0, 0.0).abs().amax(1, keepdim=True) / scale
                    z = (x / scale).clamp(-448, 448)
                    off = (y - z).abs() - half_step(z) - 1.01 * tip
                    assert (off[fine] <= 0).all(), (b, blk, float(off[fine].max()))
                if rows[0]:
                    held = cache[i, :rows[0], cols].double()
                    if scale > had:
                        same[i, :rows[0]] = False
                        kept = got[i, :rows[0], cols].double()
                        assert torch.equal(torch.nan_to_num(kept, 999.0), torch.nan_to_num(nearest(held * (had / scale)), 999.0))
                    else:
                        assert torch.equal(bits(got)[i, :rows[0], cols], bits(cache)[i, :rows[0], cols])
    assert torch.equal(bits(got)[same], bits(cache)[same])


def append_case(new, lengths, rank, rot, block, dtype, seed, grow=1.0):
    g = gen(seed)
    table, blocks = placed(lengths, block, seed)
    cache = torch.randint(0, 256, (blocks, block, rank + rot), generator=g, device="cuda", dtype=torch.uint8)
    cache[(cache & 127) == 127] = 3  # (numbers, as a block that was used holds)
    scales = torch.exp2(torch.randint(-8, -3, (blocks, 2), generator=g, device="cuda").float())
    n = sum(new)
    size = torch.exp2(torch.randint(-6, 7, (n, 1), generator=g, device="cuda").float()) * grow
    return ((randn(g, n, rank) * size).to(dtype), (3 * randn(g, n, rot) * size).to(dtype), ops.rotary_frequencies(rot),
            ints([0] + np.cumsum(new).tolist()), table, ints(lengths), cache.view(E4), scales)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("new,lengths,rank,rot,block", [
    ([1], [1], 512, 64, 16), ([1], [17], 512, 64, 16), ([1] * 7, [1, 16, 17, 31, 32, 33, 500], 512, 64, 16), ([100], [100], 512, 64, 16),
    ([5, 0, 33, 1], [5, 20, 40, 9], 256, 32, 16), ([37, 200], [39, 333], 512, 64, 12), ([64, 65, 63], [64, 65, 63], 128, 64, 64),
    ([9, 8], [1000, 8], 64, 16, 7), ([3, 4], [3, 5], 100, 6, 3), ([6], [6], 1, 2, 1), ([50, 3], [170, 70], 77, 256, 33), ([700], [1200], 512, 64, 200),
    ([1] * 150, list(range(1, 151)), 64, 32, 16), ([300, 1, 299], [300, 301, 302], 192, 64, 8)])
def test_append(new, lengths, rank, rot, block, dtype, layout):
    latent, key, f, offsets, table, n, cache, scales = append_case(new, lengths, rank, rot, block, dtype, seed=sum(new) + rank)
    before = cache.clone(), scales.clone()
    got = ops.quantized_append(latent, key, f, offsets, table, n, cache, scales, layout=layout, amplitude=1.1)
    assert got[0] is cache and got[1] is scales
    check_append(latent, key, f, offsets, table, n, before, (cache, scales), layout, 1.1)
    # again: the blocks hold these rows already, and nothing changes
    kept = cache.clone(), scales.clone()
    ops.quantized_append(latent, key, f, offsets, table, n, cache, scales, layout=layout, amplitude=1.1)
    assert torch.equal(bits(cache), bits(kept[0])) and torch.equal(scales, kept[1])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_token_by_token_with_growing_rows(dtype):
    """Every token eight times the one before: the block's rows are expressed anew at each; then ever smaller ones, which change nothing that is held."""
    g, block, rank, rot = gen(5), 16, 128, 32
    f, table = ops.rotary_frequencies(rot), ints([[2, 0]])
    cache, scales = torch.zeros(3, block, rank + rot, device="cuda").to(E4), torch.full((3, 2), 2.0 ** 50, device="cuda")
    for p in range(2 * block):
        size = 2.0 ** (3 * p - 20) if p < block else 2.0 ** (30 - 3 * p)
        latent, key = randn(g, 1, rank, dtype=dtype) * size, randn(g, 1, rot, dtype=dtype) * size
        before = cache.clone(), scales.clone()
        ops.quantized_append(latent, key, f, ints([0, 1]), table, ints([p + 1]), cache, scales)
        check_append(latent, key, f, ints([0, 1]), table, ints([p + 1]), before, (cache, scales), "interleaved")


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_append_numbers_that_are_none_and_extremes(dtype):
    """NaN and infinities are NaN and leave the scale to the others; rows of zeros take the smallest; the type's largest and smallest numbers."""
    for values in ([math.nan], [math.inf], [-math.inf, 2.0], [0.0], [torch.finfo(dtype).max], [torch.finfo(dtype).tiny], [448.0], [3.5, 3.515625, 1e-3]):
        latent, key, f, offsets, table, n, cache, scales = append_case([18], [18], 64, 16, 16, dtype, seed=3)
        latent[17], key[17] = 0.0, 0.0
        for i, v in enumerate(values):
            latent[17, 5 * i], key[17, 4 * i] = v, v
        if values[0] != values[0]:
            latent[3, 7], key[4, 2] = math.nan, math.nan
        before = cache.clone(), scales.clone()
        ops.quantized_append(latent, key, f, offsets, table, n, cache, scales)
        check_append(latent, key, f, offsets, table, n, before, (cache, scales), "interleaved")


def test_append_tables_lengths_and_offsets_out_of_range():
    """Entries outside the cache, lengths past the table and below the new tokens, offsets outside the rows: what has no place is not written."""
    latent, key, f, offsets, table, n, cache, scales = append_case([40, 30, 20, 9], [40, 50, 20, 9], 64, 16, 16, BF, seed=6)
    table[0, 1], table[1, 2] = cache.shape[0], -1
    n[2], n[3] = 5, -3  # 15 of the 20 have an index below 0; none has a place
    for o in (offsets, ints([0, 40, 70, 90, 10 ** 6]), ints([-7, 40, 70, 90, 99])):
        before = cache.clone(), scales.clone()
        ops.quantized_append(latent, key, f, o, table, n, cache, scales)
        check_append(latent, key, f, o, table, n, before, (cache, scales), "interleaved")
    n[1] = 2 ** 31 - 1  # its tokens lie past the table
    before = cache.clone(), scales.clone()
    ops.quantized_append(latent, key, f, offsets, table, n, cache, scales)
    check_append(latent, key, f, offsets, table, n, before, (cache, scales), "interleaved")
    n[1] = table.shape[1] * 16 + 10  # the last ten do
    before = cache.clone(), scales.clone()
    ops.quantized_append(latent, key, f, offsets, table, n, cache, scales)
    check_append(latent, key, f, offsets, table, n, before, (cache, scales), "interleaved")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_strides(dtype):
    """A cache that is one layer of several with a gap behind rows, inputs that are slices of one projection (also off a vector's place), rows that repeat."""
    new, lengths = [40, 1, 3], [45, 8, 3]
    latent, key, f, offsets, table, n, cache, scales = append_case(new, lengths, 512, 64, 16, dtype, seed=8)
    want = ops.quantized_append(latent, key, f, offsets, table, n, cache.clone(), scales.clone())
    for gap in (3, 8):
        both = torch.zeros(44, gap + 576 + 5, device="cuda", dtype=dtype)
        a, b = both[:, gap:gap + 512], both[:, gap + 512:gap + 576]
        a.copy_(latent), b.copy_(key)
        for left, right in ((0, 24), (16, 8), (5, 3)):
            store = torch.full((cache.shape[0], 2, 16, left + 576 + right), 7, device="cuda", dtype=torch.uint8)
            view = store[:, 1, :, left:left + 576]
            view.copy_(bits(cache))
            s = scales.clone()
            ops.quantized_append(a, b, f, offsets, table, n, view.view(E4), s)
            assert torch.equal(view, bits(want[0])) and torch.equal(s, want[1])
            view.fill_(7)
            assert (store == 7).all()
    rep = latent[:1].expand(44, 512), key[:1].expand(44, 64)
    one = [ops.quantized_append(*(t if k else t.contiguous() for t in rep), f, offsets, table, n, cache.clone(), scales.clone()) for k in (0, 1)]
    assert torch.equal(bits(one[0][0]), bits(one[1][0])) and torch.equal(one[0][1], one[1][1])


def test_append_empty():
    f = ops.rotary_frequencies(16)
    cache, scales = torch.zeros(4, 16, 80, device="cuda").to(E4), torch.ones(4, 2, device="cuda")
    e = lambda *s: torch.zeros(s, device="cuda", dtype=BF)
    ops.quantized_append(e(0, 64), e(0, 16), f, ints([0, 0]), ints([[1]]), ints([5]), cache, scales)
    ops.quantized_append(e(3, 64), e(3, 16), f, ints([0]), ints([]).reshape(0, 4), ints([]), cache, scales)
    ops.quantized_append(e(3, 64), e(3, 16), f, ints([0, 3]), ints([]).reshape(1, 0), ints([3]), cache, scales)
    assert (scales == 1).all()


# ------------------------------------------------------------- decode -----
def values_of(cache, scales, rank):
    x = cache.double()
    x[..., :rank] *= scales[:, 0, None, None].double()
    x[..., rank:] *= scales[:, 1, None, None].double()
    return x


def decode_case(lengths, new, heads, rank, key_dim, block, dtype, seed=0, junk=0x7F, spread=3):
    """Blocks of different size; rows past a request's tokens hold `junk` (NaN), and so do unused blocks with their scales."""
    g = gen(seed)
    table, blocks = placed(lengths, block, seed)
    cache = torch.full((blocks, block, rank + key_dim), junk, device="cuda", dtype=torch.uint8)
    scales = torch.full((blocks, 2), math.nan, device="cuda")
    for b, n in enumerate(lengths):
        for i in range(-(-n // block)):
            rows = min(block, n - i * block)
            x = (randn(g, rows, rank + key_dim) * 100).clamp(-448, 448).to(E4)
            cache[int(table[b, i]), :rows] = bits(x)
            scales[int(table[b, i])] = torch.exp2(torch.randint(-spread, spread, (2,), generator=g, device="cuda").float()) / 100
    q = randn(g, len(lengths), new, heads, rank + key_dim, dtype=dtype)
    return q, cache.view(E4), scales, table, ints(lengths)


def check_decode(q, cache, scales, table, lengths, rank, scale, out, lse):
    _, new, heads, width = q.shape
    u, block = U[q.dtype], cache.shape[1]
    for b, n in enumerate(lengths.tolist()):
        n = max(0, min(n, table.shape[1] * block))
        ids = table[b, :-(-n // block)].long()
        real = (ids >= 0) & (ids < cache.shape[0])
        rows = values_of(cache[ids * real], scales[ids * real].clamp(2.0 ** -60, 2.0 ** 60), rank)
        rows[~real] = 0
        rows = rows.flatten(0, 1)[:n]
        for t in range(new):
            sees = n - new + 1 + t
            if sees <= 0:
                assert not out[b, t].any() and (lse[b, t] == -math.inf).all()
                continue
            s = q[b, t].double() @ rows[:sees].T * scale
            p = torch.softmax(s, 1)
            want, mag = p @ rows[:sees, :rank], p @ rows[:sees, :rank].abs()
            tip = abs(scale) * 2.0 ** -21 * q[b, t].double().abs().amax(1, keepdim=True) * (rows[:sees].abs().sum(1).max())
            off = (out[b, t].double() - want).abs()
            assert (off <= u * want.abs() + (2 * u + 1e-5 + 2 * tip) * mag + 1e-7).all(), (b, t, float((off / mag).max()))
            want = torch.logsumexp(s, 1)
            assert ((lse[b, t].double() - want).abs() <= 1e-5 + 1e-6 * want.abs() + tip[:, 0]).all(), (b, t)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lengths,new,heads,rank,key_dim,block", [
    ([1], 1, 1, 512, 64, 16), ([0], 1, 16, 512, 64, 16), ([0, 5, 0, 1], 1, 16, 512, 64, 16), ([63, 64, 65, 127, 128, 129], 1, 16, 512, 64, 16),
    ([777], 1, 16, 512, 64, 16), ([300, 2, 1000], 1, 128, 512, 64, 16), ([200, 31], 1, 65, 512, 64, 12), ([500], 1, 64, 256, 32, 7),
    ([90, 400], 3, 16, 512, 64, 64), ([2, 5, 1], 5, 3, 512, 64, 16), ([64, 65, 66], 4, 17, 128, 64, 1), ([333], 1, 130, 512, 0, 16),
    ([1025, 17], 2, 40, 64, 16, 48), ([3000], 1, 20, 512, 64, 16), ([40] * 70, 1, 5, 192, 48, 16), ([4100, 1, 0, 2500, 64], 7, 10, 512, 64, 33),
    ([k * 7 % 90 for k in range(300)], 1, 4, 128, 64, 16), ([700, 130], 2, 96, 512, 64, 32), ([500, 0, 77], 4, 64, 256, 64, 24),
    ([6000, 40], 1, 33, 448, 32, 128), ([2049], 3, 7, 320, 64, 256), ([129, 4000], 2, 16, 384, 16, 4)])
def test_decode(lengths, new, heads, rank, key_dim, block, dtype):
    q, cache, scales, table, n = decode_case(lengths, new, heads, rank, key_dim, block, dtype, seed=len(lengths) + heads)
    scale = 1.0 / math.sqrt(rank + key_dim)
    out = torch.full((len(lengths), new, heads, rank), float("nan"), device="cuda", dtype=dtype)
    got, lse = ops.quantized_decode(q, cache, scales, table, n, scale=scale, out=out)
    assert got is out
    check_decode(q, cache, scales, table, n, rank, scale, out, lse)
    again, lse2 = ops.quantized_decode(q, cache, scales, table, n, scale=scale, out=torch.empty_like(out))
    assert torch.equal(again, out) and torch.equal(lse2, lse)  # the same bits


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lengths,new,heads,rank,key_dim,block", [
    ([100, 0, 45, 330], 40, 130, 64, 16, 16), ([90, 700], 33, 77, 128, 0, 16), ([1000], 1, 16, 512, 64, 1000), ([5000], 2, 24, 512, 64, 5003),
    ([64 * k + 1 for k in range(140)], 1, 40, 64, 64, 16)])
def test_decode_more_rows_than_blocks_of_threads_and_one_block_of_cache(lengths, new, heads, rank, key_dim, block, dtype):
    q, cache, scales, table, n = decode_case(lengths, new, heads, rank, key_dim, block, dtype, seed=heads)
    if len(lengths) == 1:  # a cache of a single block
        i = int(table[0, 0])
        cache, scales, table = cache[i:i + 1], scales[i:i + 1], torch.zeros_like(table)
    scale = 1.0 / math.sqrt(rank + key_dim)
    out, lse = ops.quantized_decode(q, cache, scales, table, n, scale=scale, out=torch.full((len(lengths), new, heads, rank), float("nan"), device="cuda", dtype=dtype))
    check_decode(q, cache, scales, table, n, rank, scale, out, lse)


def test_decode_without_a_cache_or_a_table():
    q = randn(gen(3), 2, 2, 20, 576, dtype=BF)
    none = torch.empty(0, 16, 576, device="cuda", dtype=torch.uint8).view(E4), torch.empty(0, 2, device="cuda")
    some = torch.zeros(4, 16, 576, device="cuda", dtype=torch.uint8).view(E4), torch.ones(4, 2, device="cuda")
    out, lse = ops.quantized_decode(q, *none, ints([[0, 1], [5, 2]]), ints([20, 1]), scale=0.1)  # blocks of zeros
    assert not out.any() and torch.allclose(lse[0, :, 0].cpu(), torch.log(torch.tensor([19.0, 20.0])), rtol=0, atol=1e-6)
    assert (lse[1, 0] == -math.inf).all() and (lse[1, 1] == 0).all()
    out, lse = ops.quantized_decode(q, *some, ints([]).reshape(2, 0), ints([20, 1]), scale=0.1)  # no token can be named
    assert not out.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, HF])
def test_decode_sizes_far_apart(dtype):
    """Blocks whose scales differ by 2^24 (the large ones with few of the weights), queries of very different size, negative and zero scale."""
    q, cache, scales, table, n = decode_case([700, 700], 1, 16, 512, 64, 16, dtype, seed=9, spread=12)
    size = torch.exp2(torch.arange(16, device="cuda") - 6.0)[:, None] if dtype is BF else torch.exp2(torch.arange(16, device="cuda") / 2 - 4.0)[:, None]
    q = (q.float() * size).to(dtype)
    for scale in (0.01, -0.003, 0.0):
        out, lse = ops.quantized_decode(q, cache, scales, table, n, scale=scale)
        check_decode(q, cache, scales, table, n, 512, scale, out, lse)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_decode_peaked_and_growing_scores(dtype):
    """One token far above the others; scores that grow along the cache, so that the running maximum moves at every tile."""
    q, cache, scales, table, n = decode_case([700, 900], 1, 16, 512, 64, 16, dtype, seed=10)
    f = cache.float()
    f[int(table[0, 20]), 3] = (q[0, 0, 0].float() * 60).clamp(-400, 400)
    for i in range(57):
        f[int(table[1, i])] = f[int(table[1, i])].nan_to_num(0.0) * 0.2 + q[1, 0, 1].float() * (0.25 * i)
        scales[int(table[1, i])] = 0.01
    cache = f.to(E4)
    bits(cache)[int(table[0, 43]), 12:] = 0x7F
    for scale in (0.1, -0.2):
        out, lse = ops.quantized_decode(q, cache, scales, table, n, scale=scale)
        check_decode(q, cache, scales, table, n, 512, scale, out, lse)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_decode_many_small_weights(dtype):
    """30,000 tokens of 2^-13 of the weight of one: together they outweigh it, and none may be lost."""
    q, cache, scales, table, n = decode_case([30000], 1, 8, 256, 64, 64, dtype, seed=11)
    f = torch.zeros(cache.shape, device="cuda")
    f[..., :256] = torch.randn(cache.shape[:2] + (256,), device="cuda", generator=gen(1)) * 10 + 50
    q.zero_()
    q[..., 256] = 1.0
    f[int(table[0, 7]), 5, 256] = 256.0
    f[int(table[0, 7]), 5, :256] = -30.0
    scales[:] = 1.0
    out, lse = ops.quantized_decode(q, f.to(E4), scales, table, n, scale=13 * math.log(2) / 256)
    check_decode(q, f.to(E4), scales, table, n, 256, 13 * math.log(2) / 256, out, lse)


def test_decode_scales_out_of_range():
    """Scales at and past the ends are taken as the ends, NaN as the smallest."""
    q, cache, scales, table, n = decode_case([200], 1, 4, 128, 32, 16, BF, seed=12)
    for i, s in enumerate((0.0, -1.0, 2.0 ** -60, 2.0 ** -100, math.nan)):
        scales[int(table[0, i]), i % 2] = s
    out = torch.empty(1, 1, 4, 128, device="cuda", dtype=BF)
    _, lse = ops.quantized_decode(q, cache, scales, table, n, scale=0.1, out=out)
    check_decode(q, cache, scales.nan_to_num(0.0), table, n, 128, 0.1, out, lse)
    scales[int(table[0, 7]), 0] = math.inf  # its weight times 2^60 is beyond what 16 bits hold, not beyond 32
    small, lse2 = ops.quantized_decode(q * 0, cache, scales, table, n, scale=0.1, out=torch.empty_like(out))
    assert torch.isfinite(lse2).all() and not torch.isnan(small).any()


def test_decode_table_and_lengths_out_of_range():
    q, cache, scales, table, n = decode_case([100, 90], 1, 16, 512, 64, 16, BF, seed=4, junk=0x30)
    scales = scales.nan_to_num(0.5)
    table[0, 2], table[1, 1] = cache.shape[0], 2 ** 31 - 1
    n[0] = 2 ** 31 - 1
    out, lse = ops.quantized_decode(q, cache, scales, table, n, scale=0.05)
    check_decode(q, cache, scales, table, n, 512, 0.05, out, lse)
    n[0] = -5
    out, lse = ops.quantized_decode(q, cache, scales, table, n, scale=0.05)
    assert not out[0].any() and (lse[0] == -math.inf).all()


@pytest.mark.parametrize("lengths", [[60, 40], [5000, 40]])  # whole requests, and joined parts
def test_decode_numbers_that_are_none_show(lengths):
    """NaN in a row makes all that see it NaN, NaN or an infinity in a query its own result; others keep theirs."""
    q, cache, scales, table, n = decode_case(lengths, 1, 16, 512, 64, 16, BF, seed=13)
    want, lse = ops.quantized_decode(q, cache, scales, table, n, scale=0.05)
    for bad in (math.nan, math.inf):
        p = q.clone()
        p[0, 0, 3, 100] = bad
        out, lse2 = ops.quantized_decode(p, cache, scales, table, n, scale=0.05)
        assert out[0, 0, 3].isnan().all() and lse2[0, 0, 3].isnan()
        keep = torch.ones(16, dtype=torch.bool)
        keep[3] = False
        assert torch.equal(out[0, 0, keep], want[0, 0, keep]) and torch.equal(out[1], want[1]) and torch.equal(lse2[1], lse[1])
    bits(cache)[int(table[0, 1]), 5, 100] = 0xFF
    out, lse2 = ops.quantized_decode(q, cache, scales, table, n, scale=0.05)
    assert out[0].isnan().all() and lse2[0].isnan().all()
    assert torch.equal(out[1], want[1]) and torch.equal(lse2[1], lse[1])


@pytest.mark.parametrize("lengths", [[70, 300], [128, 5], [4000, 257]])
@pytest.mark.parametrize("column", [3, 515])
def test_decode_later_tokens_stay_out_of_earlier_rows(lengths, column):
    """NaN in the newest tokens: the rows that do not see it have the bits of a call without."""
    q, cache, scales, table, n = decode_case(lengths, 4, 9, 512, 64, 16, BF, seed=14)
    want, lse = ops.quantized_decode(q, cache, scales, table, n, scale=0.05)
    for back in (1, 2, 3):  # the token that is `back` from the last
        c = cache.clone()
        p = lengths[0] - back
        bits(c)[int(table[0, p // 16]), p % 16, column] = 0x7F
        out, lse2 = ops.quantized_decode(q, c, scales, table, n, scale=0.05)
        assert torch.equal(out[0, :4 - back], want[0, :4 - back]) and torch.equal(lse2[0, :4 - back], lse[0, :4 - back])
        assert out[0, 4 - back:].isnan().all() and lse2[0, 4 - back:].isnan().all()
        assert torch.equal(out[1], want[1]) and torch.equal(lse2[1], lse[1])


def test_decode_scores_past_32_bits_and_far_down():
    """Scores beyond 2^23 keep their weights in range; all of them far below zero."""
    q, cache, scales, table, n = decode_case([300], 1, 4, 128, 16, 16, BF, seed=15)
    for scale in (3e7, -3e7):
        out, lse = ops.quantized_decode(q, cache, scales, table, n, scale=scale, out=torch.empty(1, 1, 4, 128, device="cuda", dtype=BF))
        rows = values_of(cache[table[0, :19].long()], scales[table[0, :19].long()], 128).flatten(0, 1)[:300]
        s = q[0, 0].double() @ rows.T
        best = (s * scale).argmax(1)  # (the others are more than 2^20 below)
        assert torch.isfinite(out).all()
        off = (out[0, 0].double() - rows[best, :128]).abs()
        assert (off <= U[BF] * rows[best, :128].abs() + 1e-6).all()
        assert torch.allclose(lse[0, 0].double(), (s * scale).amax(1), rtol=2e-6)


def test_decode_strides():
    q, cache, scales, table, n = decode_case([150, 40], 2, 6, 512, 64, 16, BF, seed=6)
    wide = torch.zeros(2, 2, 3, 6, 600, device="cuda", dtype=BF)
    qv = wide[:, :, 1, :, 8:584]
    qv.copy_(q)
    store = torch.full((cache.shape[0], 3, 16, 608), 0x7F, device="cuda", dtype=torch.uint8)
    cv = store[:, 2, :, 16:592]
    cv.copy_(bits(cache))
    tv = torch.zeros(2, 40, dtype=torch.int32, device="cuda")[:, 3:3 + table.shape[1]]
    tv.copy_(table)
    ov = torch.zeros(2, 6, 2, 520, device="cuda", dtype=BF).transpose(1, 2)[..., 8:]
    a, la = ops.quantized_decode(q, cache, scales, table, n, scale=0.05)
    b, lb = ops.quantized_decode(qv, cv.view(E4), scales, tv, n, scale=0.05, out=ov)
    assert torch.equal(a, b) and torch.equal(la, lb)
    for v in (q[:, :, :1].expand(q.shape), q[:1].expand(q.shape), q[:, :1].expand(q.shape)):
        a, la = ops.quantized_decode(v.contiguous(), cache, scales, table, n, scale=0.05)
        b, lb = ops.quantized_decode(v, cache, scales, table, n, scale=0.05)
        assert torch.equal(a, b) and torch.equal(la, lb)
    a, la = ops.quantized_decode(q, cache, scales, table[:1].expand(table.shape).contiguous(), n, scale=0.05)
    b, lb = ops.quantized_decode(q, cache, scales, table[:1].expand(table.shape), n, scale=0.05)
    assert torch.equal(a, b) and torch.equal(la, lb)


def test_offsets_past_32_bits():
    """A cache of more than 2^32 numbers: rows at its far end, appended and attended."""
    blocks = 480000
    cache, scales = torch.zeros(blocks, 16, 576, device="cuda", dtype=torch.uint8).view(E4), torch.ones(blocks, 2, device="cuda")
    g = gen(7)
    ids = [blocks - 1, 0, blocks - 2, 466100, 234000]
    table, n = ints([ids]), ints([77])
    latent, key = randn(g, 77, 512, dtype=BF), randn(g, 77, 64, dtype=BF)
    f = ops.rotary_frequencies(64)
    ops.quantized_append(latent, key, f, ints([0, 77]), table, n, cache, scales)
    small = torch.zeros(5, 16, 576, device="cuda", dtype=torch.uint8).view(E4), torch.ones(5, 2, device="cuda")
    ops.quantized_append(latent, key, f, ints([0, 77]), ints([[0, 1, 2, 3, 4]]), n, *small)
    assert torch.equal(bits(cache)[ids], bits(small[0])) and torch.equal(scales[ids], small[1])
    q = randn(g, 1, 1, 16, 576, dtype=BF)
    out, lse = ops.quantized_decode(q, cache, scales, table, n, scale=0.06)
    check_decode(q, cache, scales, table, n, 512, 0.06, out, lse)


# ----------------------------------------------------------- together -----
def test_on_another_stream_and_in_a_row():
    """Calls in a row, on a stream of their own, give the bits of calls with a wait after each."""
    def steps(wait):
        q, cache, scales, table, n = decode_case([600, 70, 1200], 2, 16, 512, 64, 16, BF, seed=8, junk=0)
        scales = scales.nan_to_num(1.0)
        g = gen(3)
        latent, key, f = randn(g, 6, 512, dtype=BF), randn(g, 6, 64, dtype=BF), ops.rotary_frequencies(64)
        outs = []
        for i in range(20):
            ops.quantized_append(latent * (0.5 + i % 3), key * (0.5 + i % 5), f, ints([0, 2, 4, 6]), table, n, cache, scales)
            if wait:
                torch.cuda.synchronize()
            out, lse = ops.quantized_decode(q, cache, scales, table, n, scale=0.05)
            if wait:
                torch.cuda.synchronize()
            latent[:, :] = out[:, :, 0].reshape(6, 512)
            other, _ = ops.quantized_decode(q, cache, scales, table, n - 1, scale=0.05)
            q[..., :512] = 0.5 * (q[..., :512] + other)
            outs.append(lse)
        return [q, bits(cache), scales, torch.stack(outs)]
    want = steps(True)
    assert all(torch.isfinite(t).all() for t in want)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        got = steps(False)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_in_a_graph_with_other_lengths():
    """Captured once, replayed with other lengths, rows and tables; two graphs replayed side by side keep their results."""
    q, cache, scales, table, n = decode_case([600, 1200], 1, 32, 512, 64, 16, BF, seed=8, junk=0)
    scales = scales.nan_to_num(1.0)
    latent, key, f, o = randn(gen(1), 2, 512, dtype=BF), randn(gen(2), 2, 64, dtype=BF), ops.rotary_frequencies(64), ints([0, 1, 2])

    def call(cache, scales):
        ops.quantized_append(latent, key, f, o, table, n, cache, scales)
        return ops.quantized_decode(q, cache, scales, table, n, scale=0.05)

    call(cache.clone(), scales.clone())
    made, places = [], [(cache.clone(), scales.clone()) for _ in range(2)]
    for c, s in places:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            made.append((graph, call(c, s)))
    q.mul_(2), n.copy_(ints([301, 999])), latent.mul_(3)
    for c, s in places:
        c.view(torch.uint8).copy_(bits(cache)), s.copy_(scales)
    fresh = cache.clone(), scales.clone()
    want = [t.clone() for t in (*call(*fresh), bits(fresh[0]), fresh[1])]
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (graph, _) in zip(streams, made):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for (_, got), (c, s) in zip(made, places):
        assert all(torch.equal(a, b) for a, b in zip((*got, bits(c), s), want))


def test_what_autograd_sees():
    q, cache, scales, table, n = decode_case([9], 1, 4, 512, 64, 16, BF, seed=4, junk=0)
    latent, key, f = randn(gen(1), 1, 512, dtype=BF), randn(gen(2), 1, 64, dtype=BF), ops.rotary_frequencies(64)
    out, lse = torch.empty(1, 1, 4, 512, device="cuda", dtype=BF), torch.empty(1, 1, 4, device="cuda")
    before = [t._version for t in (cache, scales, out, lse)]
    ops.quantized_append(latent, key, f, ints([0, 1]), table, n, cache, scales)
    ops.quantized_decode(q, cache, scales, table, n, scale=1.0, out=out, lse=lse)
    assert all(t._version > v for t, v in zip((cache, scales, out, lse), before))
    for bad in (latent, key):
        args = [t.clone().requires_grad_() if t is bad else t for t in (latent, key)]
        with pytest.raises(ValueError, match="forward only"):
            ops.quantized_append(*args, f, ints([0, 1]), table, n, cache, scales)
    with pytest.raises(ValueError, match="forward only"):
        ops.quantized_decode(q.clone().requires_grad_(), cache, scales, table, n, scale=1.0)
    with pytest.raises(ValueError, match="forward only"):
        ops.quantized_decode(q, cache, scales.clone().requires_grad_(), table, n, scale=1.0)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(q, torch.ones_like(q))
        with pytest.raises(ValueError, match="tangent"):
            ops.quantized_decode(dual, cache, scales, table, n, scale=1.0)
