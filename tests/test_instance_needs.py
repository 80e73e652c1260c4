"""What an instance needs besides its state: device memory to be made, work on the host for an iteration."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance  # noqa: E402
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_state import bookkeeping  # noqa: E402


@pytest.mark.gpu
@pytest.mark.parametrize("quantized", [False, True])
def test_a_cache_is_made_in_its_own_memory(quantized):
    """A cache of 1 GB (0.5 GB in 8 bits): nothing of its size is held on the way (the weights and what they are made from are 40 MB)."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    torch.cuda.empty_cache()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    node = instance.Instance(instance.Shape(layers=2, hidden=512, heads=8, vocab=4000), blocks=30000, block_tokens=16, quantized=quantized)
    size = node.cache.numel() * node.cache.element_size()
    assert node.cache.dtype is (ops.EIGHT if quantized else torch.bfloat16) and size > 5e8
    assert not node.cache.view(torch.uint8).any()
    assert torch.cuda.max_memory_allocated() - before < 1.2 * size


class Counted(list):
    """A request's blocks that count how many of them are looked at."""
    looks = 0

    def __getitem__(self, i):
        Counted.looks += 1
        return super().__getitem__(i)

    def __iter__(self):
        raise AssertionError("all of a request's blocks are gone through")

    def __array__(self, *args, **more):
        raise AssertionError("all of a request's blocks are gone through")


@pytest.mark.parametrize("new", [1, 5])
def test_new_tokens_places_take_no_look_at_the_other_blocks(new):
    held, lengths = [Counted(range(700, 800)), Counted([9, 3]), [20, 7, 2], [5]], [1590, 19, 40, 3]
    Counted.looks = 0
    positions, slots = instance._places(held, lengths, 2, new, 16)
    assert Counted.looks == 2 * new
    want = [(b, p) for b, n, k in zip(held, lengths, [new, new, 40, 3]) for p in range(n - k, n)]
    assert positions == [p for _, p in want] and slots == [list.__getitem__(b, p // 16) * 16 + p % 16 for b, p in want]


def test_blocks_are_gone_through_only_where_some_are_shared():
    node = bookkeeping(20, 4, [9, 8])
    blocks = [Counted(q.blocks) for q in node.running.values()]
    Counted.looks = 0
    assert node._own(blocks, [9, 8], 3)[1:] == (3, []) and Counted.looks == 0


def test_refused_calls_leave_the_count_of_shared_blocks(monkeypatch):
    monkeypatch.setattr(instance.Instance, "_copy", lambda self, pairs, other=None: None)
    node, other = bookkeeping(7, 4, [9, 8]), bookkeeping(2, 4, [3])
    node.fork(1), node.fork(0)
    kept = dict(node.shared)
    assert kept == {b: 1 for b in node.running[1].blocks + node.running[0].blocks[:2]}
    drafts = torch.zeros(4, 20, dtype=torch.int64)
    for call, error in ((lambda: node.fork(0, 2), RuntimeError), (lambda: node.fork(1, 9), ValueError), (lambda: node.migrate(1, other), RuntimeError),
                        (lambda: node.rewind(0, 10), ValueError), (lambda: node.iterate([torch.zeros(40, dtype=torch.int64)]), RuntimeError),
                        (lambda: node.speculate(drafts), RuntimeError), (lambda: node.speculate(drafts[:3]), ValueError)):
        with pytest.raises(error):
            call()
        assert node.shared == kept and not other.shared


@pytest.mark.gpu
@pytest.mark.parametrize("quantized", [False, True])
def test_no_copy_to_the_device_waits_for_the_layers(quantized, monkeypatch):
    """Every copy of host numbers comes before the iteration's first kernel on the cache; one of them made later would wait for all that is queued."""
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    node = instance.Instance(instance.Shape(layers=2, hidden=512, heads=8, vocab=4000), blocks=40, block_tokens=16, quantized=quantized)
    prompt = lambda n: torch.arange(n, device="cuda")
    node.iterate([prompt(20)])
    done, tensor, rotary = [], torch.tensor, ops.rotary
    monkeypatch.setattr(torch, "tensor", lambda *a, **k: (done.append("copy"), tensor(*a, **k))[1])
    monkeypatch.setattr(ops, "rotary", lambda *a, **k: (done.append("kernel"), rotary(*a, **k))[1])
    drafts = torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    for call in (lambda: node.iterate([prompt(30)]), lambda: node.iterate(), lambda: node.speculate(drafts)):
        done.clear()
        call()
        assert "copy" in done and "copy" not in done[done.index("kernel"):]
