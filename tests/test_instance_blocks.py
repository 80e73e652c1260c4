"""Shared, moved and compacted blocks of an instance, its 8-bit cache, and
iterations with drafted tokens: the operators run together as they would be used."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance  # noqa: E402
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_state import bookkeeping, state  # noqa: E402

SHAPE = dict(layers=2, hidden=512, heads=8, vocab=4000)


def whole(node, blocks):
    """Every block is free or held, and counted as often as it is held."""
    held = [b for q in node.running.values() for b in q.blocks]
    assert sorted(set(held) | set(node.free)) == list(range(blocks)) and not set(held) & set(node.free)
    assert len(set(node.free)) == len(node.free)
    assert {b: held.count(b) - 1 for b in set(held) if held.count(b) > 1} == node.shared
    for q in node.running.values():
        assert len(q.blocks) == node.blocks_for(q.length) and len(set(q.blocks)) == len(q.blocks)


@pytest.fixture
def no_copies(monkeypatch):
    """Bookkeeping without a device: what is copied is noted."""
    done = []
    monkeypatch.setattr(instance.Instance, "_copy", lambda self, pairs, other=None: done.append((list(pairs), other)))
    return done


def test_fork_shares_full_blocks_and_copies_the_last(no_copies):
    node = bookkeeping(20, 4, [9, 8])
    last = node.running[0].blocks[-1]
    ids = node.fork(0, 2)
    assert ids == [2, 3] and [node.running[i].length for i in ids] == [9, 9]
    assert all(node.running[i].blocks[:2] == node.running[0].blocks[:2] for i in ids)
    assert [a for a, _ in no_copies[0][0]] == [last, last] and len({node.running[i].blocks[2] for i in (0, 2, 3)}) == 3
    assert node.fork(1) == [4] and node.running[4].blocks == node.running[1].blocks and no_copies[1][0] == []  # a full block: shared
    whole(node, 20)
    for r in (0, 4, 2, 1, 3):
        node.release(r)
        whole(node, 20)
    assert not node.shared and len(node.free) == 20


def test_refused_forks_and_moves_change_nothing(no_copies):
    node, other = bookkeeping(5, 4, [9, 8]), bookkeeping(2, 4, [3])
    for call, error in ((lambda: node.fork(0, 0), ValueError), (lambda: node.fork(0, 7), ValueError), (lambda: node.fork(0), RuntimeError),
                        (lambda: node.migrate(0, node), ValueError), (lambda: node.migrate(0, other), RuntimeError),
                        (lambda: node.migrate(0, bookkeeping(20, 8, [])), ValueError), (lambda: node.migrate(0, bookkeeping(20, 4, [1] * 8)), ValueError)):
        before = state(node), state(other)
        with pytest.raises(error):
            call()
        assert (state(node), state(other)) == before and not no_copies


def test_a_shared_block_is_copied_before_it_is_written():
    node = bookkeeping(6, 4, [8])
    node.running[1] = instance.Running(list(node.running[0].blocks), 8, node.running[0].token)
    node.shared = {b: 1 for b in node.running[0].blocks}
    node._next = 2
    node.rewind(0, 6)
    node.rewind(1, 7)
    whole(node, 6)
    blocks, taken = node._plan([node.running[r].blocks for r in (0, 1)], [7, 8])
    blocks, taken, copies = node._own(blocks, [6, 7], taken)
    assert taken == 1 and copies == [(node.running[0].blocks[1], blocks[0][1])] and blocks[1] == node.running[1].blocks
    node.free = []
    with pytest.raises(RuntimeError, match="share"):
        node._own([list(q.blocks) for q in node.running.values()], [6, 7], 0)


def test_compact(no_copies):
    node = bookkeeping(20, 4, [9, 8, 3, 17])
    node.fork(0)
    node.release(1), node.release(2)
    used = {b for q in node.running.values() for b in q.blocks}
    no_copies.clear()
    moved = node.compact()
    pairs = no_copies[0][0]
    assert moved == len(pairs) == sum(b >= len(used) for b in used)
    assert all(a >= len(used) > b for a, b in pairs) and len({b for _, b in pairs}) == moved
    whole(node, 20)
    assert {b for q in node.running.values() for b in q.blocks} == set(range(len(used)))
    assert node.compact() == 0


# ---------------------------------------------------------------- GPU -----
def make(quantized, blocks=120, seed=0, **more):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    return instance.Instance(instance.Shape(**SHAPE), blocks=blocks, block_tokens=16, max_batch=12, quantized=quantized, seed=seed, **more)


def tokens(n, seed):
    return torch.randint(0, 4000, (n,), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def go(node, n, u=0.4):
    """n iterations of all running requests: their tokens and log-probabilities."""
    got = []
    for _ in range(n):
        _, t, lp = node.iterate(uniform=torch.full((len(node.running),), u, device="cuda"))
        got.append((t, lp))
    return torch.stack([t for t, _ in got]), torch.stack([lp for _, lp in got])


@pytest.mark.gpu
def test_the_8_bit_cache_decodes_as_the_16_bit_one():
    """A cached number is rounded by up to 2^-4 of itself, and a score of 200 tokens by a
    hundredth; log-probabilities of the same token agree to a tenth and most draws fall on the same."""
    nodes = [make(q) for q in (False, True)]
    assert nodes[1].cache.dtype is ops.EIGHT and nodes[1].scales.shape == (2, 120, 2)
    prompts = [tokens(n, n) for n in (1, 15, 16, 33, 200)]
    first = [node.iterate(prompts, uniform=torch.full((5,), 0.4, device="cuda")) for node in nodes]
    assert torch.equal(first[0][1], first[1][1])  # a prompt's own rows are not read from the cache
    (a, la), (b, lb) = (go(node, 1) for node in nodes)
    same = a == b
    assert int(same.sum()) >= 4 and torch.allclose(la[same], lb[same], atol=0.1)
    for node in nodes:
        go(node, 20)
        whole(node, 120)
    assert ops.faults() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("quantized", [False, True])
def test_forks_go_on_as_the_request_would(quantized):
    """A fork draws what its parent draws from the same numbers (their cached rows are the same bytes), and writes nothing that its parent reads."""
    node = make(quantized)
    node.iterate([tokens(40, 1), tokens(32, 2)])
    go(node, 3)
    more = node.fork(0, 2) + node.fork(1)
    whole(node, 120)
    t, lp = go(node, 20)
    order = list(node.running)
    for parent, child in ((0, more[0]), (0, more[1]), (1, more[2])):
        i, j = order.index(parent), order.index(child)
        assert torch.equal(t[:, i], t[:, j]) and torch.equal(lp[:, i], lp[:, j])
    whole(node, 120)
    node.rewind(more[0], 33)  # back into a block that it shares: writing copies it
    node.rewind(0, 33)
    go(node, 2)
    whole(node, 120)
    for r in list(node.running):
        node.release(r)
    assert len(node.free) == 120 and not node.shared


@pytest.mark.gpu
@pytest.mark.parametrize("quantized", [False, True])
def test_moved_requests_go_on_as_they_would_have(quantized):
    """Migrated to another instance, or compacted: the same tokens and log-probabilities, to the bit."""
    def run(move):
        node, other = make(quantized), make(quantized, blocks=70)
        node.iterate([tokens(50, 1), tokens(100, 2), tokens(7, 3)], uniform=torch.full((3,), 0.4, device="cuda"))
        node.release(1)
        go(node, 4)
        node.release(0)  # one request, the last blocks of those that were used
        if move == "migrate":
            other.iterate([tokens(30, 5)])
            other.release(0)
            there = node.migrate(2, other)
            assert not node.running and len(node.free) == 120 and list(other.running) == [there]
            node = other
        elif move == "compact":
            assert node.compact() == 1 and node.running[2].blocks == [0]
        t, lp = go(node, 30)
        whole(node, len(node.free) + sum(len(q.blocks) for q in node.running.values()))
        return t, lp
    want = run(None)
    for move in ("migrate", "compact"):
        got = run(move)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
@pytest.mark.parametrize("quantized", [False, True])
def test_drafted_tokens(quantized):
    """Greedy drafts of the instance itself are accepted but for near ties (several new tokens run in other
    matrix shapes than one), a wrong one is refused where it stands, and the cache is back at what was accepted."""
    node = make(quantized)
    zero = lambda n: dict(uniform=torch.zeros(n, device="cuda"), temperature=torch.zeros(n, device="cuda"))
    node.iterate([tokens(n, n) for n in (20, 31, 100)], **zero(3))
    lengths = [node.running[r].length for r in range(3)]
    kept = [node.running[r].token.clone() for r in range(3)]
    drafts = torch.stack([node.iterate(**zero(3))[1] for _ in range(4)], 1)
    for r in range(3):
        node.rewind(r, lengths[r])
        node.running[r].token = kept[r]
    drafts[1, 2] = (drafts[1, 2] + 1) % 4000
    u = dict(uniform=torch.zeros(3, 5, device="cuda"), temperature=torch.zeros(3, device="cuda"))
    ids, got, counts, lp = node.speculate(drafts, **u)
    assert ids == [0, 1, 2] and counts[1] <= 3 and sum(counts) >= 9
    for r in range(3):
        assert torch.equal(got[r, :counts[r] - 1], drafts[r, :counts[r] - 1]) and (got[r, counts[r]:] == -1).all()
        assert node.running[r].length == lengths[r] + counts[r] and int(node.running[r].token) == int(got[r, counts[r] - 1])
    whole(node, 120)
    _, none, counts, _ = node.speculate(drafts[:, :0])  # no drafts: a token each
    assert counts == [1, 1, 1] and none.shape == (3, 1)
    # with a draft's distribution, drawn from and given
    draft = torch.randn(3, 4, 4000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    guess = torch.multinomial(torch.softmax(draft.flatten(0, 1).float(), 1), 1).view(3, 4)
    before = [node.running[r].length for r in range(3)]
    _, got, counts, lp = node.speculate(guess, draft=draft)
    assert all(node.running[r].length == before[r] + counts[r] for r in range(3)) and torch.isfinite(lp[got >= 0]).all()
    go(node, 3)
    whole(node, 120)
    before = state(node)
    with pytest.raises(ValueError):
        node.speculate(drafts[:2])
    with pytest.raises(ValueError):
        node.speculate(drafts, uniform=torch.zeros(3, 4, device="cuda"))
    with pytest.raises(RuntimeError, match="out of cache blocks"):
        node.speculate(torch.zeros(3, 60, dtype=torch.int64, device="cuda").repeat(1, 20))
    assert state(node) == before
    assert ops.faults() == 0


@pytest.mark.gpu
def test_drafted_tokens_outside_the_vocabulary_are_refused():
    node = make(False)
    node.iterate([tokens(n, n) for n in (20, 31, 100)])
    drafts = torch.tensor([[5, -1, 7], [4000, 5, 6], [2 ** 40, -2 ** 63, 3]], device="cuda")
    _, got, counts, lp = node.speculate(drafts, uniform=torch.zeros(3, 4, device="cuda"))
    assert counts == [2, 1, 1] and int(got[0, 0]) == 5
    assert ((got >= 0) & (got < 4000)).sum(1).tolist() == counts and torch.isfinite(lp[got >= 0]).all()
    whole(node, 120)


@pytest.mark.gpu
def test_times_of_an_instance_with_an_8_bit_cache():
    node = make(True)
    samples = instance.measure(node, prefill_tokens=(0, 64), decodes=(0, 4, 10), context=60, repeats=1)
    assert len(samples) == 5 and all(t > 0 and math.isfinite(t) for _, _, t in samples) and not node.running
