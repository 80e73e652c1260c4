"""Copies of cache blocks on the GPU: every byte of what is copied, and no other."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402

pytestmark = pytest.mark.gpu

BF, F32, E4 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def filled(g, shape, dtype):
    n = torch.empty(0, dtype=dtype).element_size()
    return torch.randint(0, 256, (*shape[:-1], shape[-1] * n), generator=g, device="cuda", dtype=torch.uint8).view(dtype)


def raw(t):
    return t.view(torch.uint8) if t.is_contiguous() else t.contiguous().view(torch.uint8)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def expected(source, destination, pairs):
    want = raw(destination).clone()
    for a, b in pairs:
        if 0 <= a < source.shape[1] and 0 <= b < destination.shape[1]:
            want[:, b] = raw(source)[:, a]
    return want


@pytest.mark.parametrize("dtype", [BF, F32, E4, torch.uint8, torch.int64])
@pytest.mark.parametrize("layers,have,room,block,pairs", [
    (1, 1, 1, (16, 576), 1), (2, 30, 20, (16, 576), 9), (27, 64, 64, (12, 560), 20), (3, 40, 50, (2,), 33), (1, 9, 9, (1, 1), 7), (5, 300, 300, (7, 33), 140),
    (60, 20, 30, (64, 40), 10), (2, 2000, 2100, (3,), 2000), (4, 12, 12, (200, 576), 6), (1, 5000, 5000, (16, 8), 4000)])
def test_between_two(layers, have, room, block, pairs, dtype):
    g = torch.Generator(device="cuda").manual_seed(pairs)
    source, destination = filled(g, (layers, have, *block), dtype), filled(g, (layers, room, *block), dtype)
    a = torch.randint(0, have, (pairs,), generator=g, device="cuda", dtype=torch.int32)  # some read more than once
    b = torch.randperm(room, generator=g, device="cuda")[:pairs].int()
    if pairs > 5:
        a[2], b[3], a[4], b[4] = have, room, -1, 2 ** 31 - 1
    want = expected(source, destination, list(zip(a.tolist(), b.tolist())))
    kept = raw(source).clone()
    version = destination._version
    assert ops.block_copy(source, destination, a, b) is destination
    assert torch.equal(raw(destination), want) and torch.equal(raw(source), kept) and destination._version > version


@pytest.mark.parametrize("dtype", [BF, E4, F32])
def test_within_one(dtype):
    """Blocks at the end of a cache into free ones at its start."""
    g = torch.Generator(device="cuda").manual_seed(1)
    cache = filled(g, (3, 500, 16, 80), dtype)
    order = torch.randperm(500, generator=g, device="cuda").int()
    a, b = order[:240].clone(), order[250:490].clone()
    b[::7] = -1
    want = expected(cache, cache, list(zip(a.tolist(), b.tolist())))
    ops.block_copy(cache, cache, a, b)
    assert torch.equal(raw(cache), want)


@pytest.mark.parametrize("dtype", [BF, E4])
@pytest.mark.parametrize("first,width,gap", [(0, 576, 0), (3, 573, 24), (16, 560, 24), (5, 33, 1), (8, 64, 8)])
def test_strides(dtype, first, width, gap):
    """Layers inside blocks, rows with gaps, parts of rows: nothing around them is written; layers that repeat are read."""
    g = torch.Generator(device="cuda").manual_seed(2)
    store, room = filled(g, (20, 4, 16, first + width + gap), dtype), filled(g, (15, 4, 18, first + width + gap), dtype)
    source, destination = store.transpose(0, 1)[..., first:first + width], room.transpose(0, 1)[:, :, 1:17, first:first + width]
    a, b = ints([0, 19, 7, 7, 3]), ints([14, 0, 5, 6, 1])
    want, e = raw(room).clone(), room.element_size()
    for x, y in zip(a.tolist(), b.tolist()):
        want[y, :, 1:17, e * first:e * (first + width)] = raw(store)[x, :, :, e * first:e * (first + width)]
    ops.block_copy(source, destination, a, b)
    assert torch.equal(raw(room), want)
    one = source[:1].expand(4, -1, -1, -1)
    other = [torch.zeros_like(destination.contiguous()) for _ in range(2)]
    ops.block_copy(one, other[0], a, b), ops.block_copy(one.contiguous(), other[1], a, b)
    assert torch.equal(raw(other[0]), raw(other[1]))


def test_dimensions_of_one_and_empty():
    g = torch.Generator(device="cuda").manual_seed(3)
    source = filled(g, (1, 1, 1, 64), BF)
    destination = torch.zeros(1, 1, 1, 64, device="cuda", dtype=BF)
    ops.block_copy(source.as_strided((1, 1, 1, 64), (3, 5, 7, 1)), destination.as_strided((1, 1, 1, 64), (1, 1, 1, 1)), ints([0]), ints([0]))
    assert torch.equal(raw(source), raw(destination))
    for shape, n in (((0, 5, 4), 1), ((2, 0, 4), 1), ((2, 5, 0), 1), ((2, 5, 0, 4), 1), ((2, 5, 4), 0)):
        t = torch.zeros(shape, device="cuda")
        ops.block_copy(t, t.clone(), ints([0] * n), ints([1] * n))


def test_offsets_past_32_bits():
    g = torch.Generator(device="cuda").manual_seed(4)
    cache = torch.zeros(2, 300000, 16, 576, device="cuda", dtype=torch.uint8)
    for i in (0, 299999, 150000):
        cache[:, i] = torch.randint(0, 256, (2, 16, 576), generator=g, device="cuda", dtype=torch.uint8)
    ops.block_copy(cache, cache, ints([0, 299999, 150000]), ints([299998, 1, 233333]))
    for a, b in ((0, 299998), (299999, 1), (150000, 233333)):
        assert torch.equal(cache[:, a], cache[:, b]) and cache[:, b].any()
    assert int(cache.view(2, 300000, -1)[0].any(1).sum()) == 6


def test_streams_graphs_and_order():
    """A chain of copies in a row gives what it gives with waits between; captured, it follows its lists."""
    g = torch.Generator(device="cuda").manual_seed(5)
    first = filled(g, (4, 64, 16, 96), E4)
    moves = [torch.randperm(64, generator=g, device="cuda").int() for _ in range(12)]

    def steps(wait):
        cache = first.clone()
        for m in moves:
            ops.block_copy(cache, cache, m[:30], m[32:62])
            if wait:
                torch.cuda.synchronize()
        return raw(cache).clone()
    want = steps(True)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
        got = steps(False)
    s.synchronize()
    assert torch.equal(got, want)
    cache, a, b = first.clone(), moves[0][:30].clone(), moves[0][32:62].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.block_copy(cache, cache, a, b)
    cache.view(torch.uint8).copy_(raw(first))
    a.copy_(moves[1][:30]), b.copy_(moves[1][32:62])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(raw(cache), expected(first, first, list(zip(a.tolist(), b.tolist()))))


def test_gradients_are_refused():
    t = torch.zeros(2, 5, 4, device="cuda")
    with pytest.raises(ValueError, match="forward only"):
        ops.block_copy(t.clone().requires_grad_(), t, ints([0]), ints([1]))
