"""What an instance needs besides its state: device memory to be made, work on the host for an iteration."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance  # noqa: E402
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402


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
