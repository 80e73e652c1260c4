"""What the timed iterations of ``instance.measure`` hold, and what it leaves behind."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance  # noqa: E402
from test_instance_state import bookkeeping, state  # noqa: E402


def test_rewind_gives_blocks_back():
    node = bookkeeping(10, 4, [9, 3])
    free = list(node.free)
    node.rewind(0, 8)
    assert node.running[0].length == 8 and node.running[0].blocks == [0, 1] and node.free == free + [2]
    node.rewind(0, 8)
    for tokens in (0, 9):
        with pytest.raises(ValueError, match="go back"):
            node.rewind(0, tokens)
    assert state(node)[2] == {0: ([0, 1], 8), 1: ([3], 3)}


class Recorded(instance.Instance):
    """Keeps (lengths before, prompt lengths) of every iteration that advances."""

    def iterate(self, prompts=(), *, advance=True, **rest):
        before = [q.length for q in self.running.values()]
        out = super().iterate(prompts, advance=advance, **rest)
        if advance:
            self.log.append((before, [len(p) for p in prompts]))
        return out


@pytest.fixture(scope="module")
def node():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    node = Recorded(instance.Shape(layers=2, hidden=512, heads=8, vocab=4000), blocks=40, block_tokens=16, max_batch=12)
    node.log = []
    return node


@pytest.mark.gpu
def test_every_timed_iteration_has_the_context_that_is_named(node):
    """40 blocks of 16; 63 cached tokens and the new one take 4 blocks a request."""
    samples = instance.measure(node, prefill_tokens=(0, 64, 80, 320, 336), decodes=(0, 5, 9, 11, 13), context=63, repeats=2)
    want = [(64, 0), (80, 0), (320, 0), (336, 0), (0, 5), (64, 5), (80, 5), (320, 5), (0, 9), (64, 9)]
    assert [s[:2] for s in samples] == want and all(t > 0 for _, _, t in samples)
    assert node.log == [([63] * d, [p] * (p > 0)) for p, d in want for _ in range(3)]
    assert not node.running and sorted(node.free) == list(range(40))


@pytest.mark.gpu
def test_nothing_stays_behind_when_an_iteration_raises(node):
    def broken(x):
        if len(node.running) == 4:
            raise KeyError("feed_forward")
        return x

    node.feed_forward = broken
    with pytest.raises(KeyError):
        instance.measure(node, prefill_tokens=(0, 16), decodes=(4,), context=20, repeats=1)
    node.feed_forward = None
    assert not node.running and sorted(node.free) == list(range(40))
    for bad in (dict(context=0), dict(repeats=0)):
        with pytest.raises(ValueError):
            instance.measure(node, **bad)
