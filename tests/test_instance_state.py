"""What an instance keeps between iterations when a call is refused."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance  # noqa: E402


def state(node):
    return list(node.free), node._next, {r: (list(q.blocks), q.length) for r, q in node.running.items()}


def bookkeeping(blocks, block_tokens, lengths, max_batch=8):
    """An instance's bookkeeping alone, with running requests of the given lengths (no device, no weights)."""
    node = object.__new__(instance.Instance)
    node.shape, node.block_tokens, node.max_batch = instance.Shape(), block_tokens, max_batch
    node.free, node.running, node._next = list(range(blocks))[::-1], {}, len(lengths)
    for r, n in enumerate(lengths):
        node.running[r] = instance.Running([node.free.pop() for _ in range(-(-n // block_tokens))], n, torch.zeros(1, dtype=torch.int64))
    return node


def test_an_iteration_that_does_not_fit_changes_nothing():
    """Running requests of 48 (a block more is needed) and 7 tokens, a prompt that fits and one that does not."""
    node = bookkeeping(200, 16, [48, 7])
    before = state(node)
    prompts = [torch.zeros(n, dtype=torch.int64) for n in (33, 4000)]
    with pytest.raises(RuntimeError, match="out of cache blocks"):
        node.iterate(prompts)
    assert state(node) == before
    with pytest.raises(RuntimeError, match="out of cache blocks: 1 wanted, 0 free"):
        full = bookkeeping(4, 16, [48, 7])
        full.iterate()
    assert state(full) == state(bookkeeping(4, 16, [48, 7]))


def test_a_plan_takes_blocks_from_the_end_of_the_free_list():
    node = bookkeeping(10, 4, [4, 3])
    blocks, taken = node._plan([node.running[0].blocks, node.running[1].blocks, []], [5, 4, 9])
    assert blocks == [[0, 2], [1], [3, 4, 5]] and taken == 4 and node.free == [9, 8, 7, 6, 5, 4, 3, 2]


@pytest.mark.gpu
def test_refused_iterations_leave_the_tokens_as_they_would_have_been():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    g = torch.Generator(device="cuda").manual_seed(3)
    prompts = [torch.randint(0, 4000, (n,), generator=g, device="cuda") for n in (48, 7, 20)]
    half = lambda n: torch.full((n,), 0.5, device="cuda")

    def broken(x):
        raise KeyError("feed_forward")

    def run(refuse):
        node = instance.Instance(instance.Shape(layers=2, hidden=512, heads=8, vocab=4000), blocks=20, block_tokens=16, max_batch=6)
        drawn = [node.iterate(prompts[:2], uniform=half(2))[1]]
        for i in range(4):
            if refuse:
                before = state(node)
                with pytest.raises(RuntimeError, match="out of cache blocks"):
                    node.iterate([prompts[2], prompts[0].repeat(9)])
                with pytest.raises(ValueError):  # one value too few: refused by the last operator
                    node.iterate([prompts[2]], uniform=half(2 + (i > 1)))
                node.feed_forward = broken
                with pytest.raises(KeyError):
                    node.iterate([prompts[2]])
                node.feed_forward = None
                assert state(node) == before
            drawn.append(node.iterate([prompts[2]] if i == 1 else [], uniform=half(2 + (i >= 1)))[1])
        return drawn, state(node)

    want, kept = run(False)
    got, kept2 = run(True)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and kept == kept2
