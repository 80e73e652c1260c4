"""The fit of iteration times and their way into a workload (CPU), and an
instance whose iterations run the operators together (GPU)."""
import numpy as np
import pytest

from paper_2608_16336_gb300 import workloads

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance, mtsim  # noqa: E402


def test_fit_recovers_the_model():
    samples = [(p, d, 4000.0 + 20 * p + 30 * d) for p in (0, 100, 1000) for d in (0, 8, 64) if p or d]
    assert instance.fit_iteration_times(samples) == (4000, 20, 30)


def test_fit_keeps_constants_at_or_above_zero():
    samples = [(p, d, 500.0 + 3 * p - 0.5 * d) for p in (0, 100, 1000) for d in (1, 8, 64)]
    base, a, b = instance.fit_iteration_times(samples)
    assert b == 0 and a == 3 and 450 < base < 520
    with pytest.raises(ValueError):
        instance.fit_iteration_times(samples[:2])
    with pytest.raises(ValueError):
        instance.fit_iteration_times([(0, 1, 0.0)] * 4)


def test_times_enter_the_workload():
    w = workloads.config(0, requests=20)
    v = instance.with_times(w, (1234, 5, 6))
    assert (v.iter_base_us, v.iter_us_per_prefill_token, v.iter_us_per_decode_seq) == (1234, 5, 6)
    assert w.iter_base_us == 4000 and v.arrival_us is w.arrival_us


@pytest.fixture(scope="module")
def node():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    shape = instance.Shape(layers=2, hidden=512, heads=8, vocab=4000)
    return instance.Instance(shape, blocks=200, block_tokens=16, max_batch=12)


def tokens(n, seed):
    return torch.randint(0, 4000, (n,), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.gpu
def test_decoding_continues_a_prefill(node):
    """A token's distribution after prefill + decode (absorbed form over the
    cache) is that after a prefill of the longer prompt (expanded form):
    both round their operands to bfloat16, so log-probabilities agree to a few hundredths."""
    zero = lambda n: torch.zeros(n, device="cuda")
    greedy = lambda n: dict(uniform=zero(n), temperature=zero(n))
    lengths = (1, 15, 16, 33, 200)
    prompts = [tokens(n, n) for n in lengths]
    first, drawn, _ = node.iterate(prompts, **greedy(len(prompts)))
    ids, _, lp = node.iterate(uniform=torch.full((5,), 0.4, device="cuda"))
    assert ids == first
    token = torch.cat([node.running[r].token for r in ids])
    for r in ids:
        node.release(r)
    longer = [torch.cat((p, drawn[i:i + 1])) for i, p in enumerate(prompts)]
    again, token2, lp2 = node.iterate(longer, uniform=torch.full((5,), 0.4, device="cuda"))
    for r in again:
        node.release(r)
    assert len(node.free) == 200 and not node.running
    # near ties in the draw may fall either way; most must agree, and where they do so must the probabilities
    same = token == token2
    assert int(same.sum()) >= 3
    assert torch.allclose(lp[same], lp2[same], atol=0.1), (lp, lp2)


@pytest.mark.gpu
def test_mixed_iterations_and_blocks(node):
    a, _, _ = node.iterate([tokens(40, 1), tokens(7, 2)])
    b, t, lp = node.iterate([tokens(100, 3)])
    assert b == a + [b[-1]] and t.shape == (3,) and bool((lp <= 0).all()) and bool(((t >= 0) & (t < 4000)).all())
    assert [node.running[r].length for r in b] == [41, 8, 100]
    for _ in range(9):
        node.iterate()
    assert [len(node.running[r].blocks) for r in b] == [4, 2, 7]  # 50, 17 and 109 tokens of 16 a block
    used = [x for r in b for x in node.running[r].blocks]
    assert len(set(used)) == len(used) and len(node.free) == 200 - 13
    with pytest.raises(ValueError, match="max_batch"):
        node.iterate([tokens(1, 1)] * 10)
    with pytest.raises(RuntimeError, match="out of cache blocks"):
        node.iterate([tokens(4000, 1)])
    for r in list(node.running):
        node.release(r)
    node.free = sorted(node.free)[::-1]
    assert len(set(node.free)) == 200


@pytest.mark.gpu
def test_measured_times_drive_a_simulation(node):
    samples = instance.measure(node, prefill_tokens=(0, 64, 512), decodes=(0, 4, 10), context=60, repeats=2)
    assert len(samples) == 8 and all(t > 0 for _, _, t in samples)
    times = instance.fit_iteration_times(samples)
    w = instance.with_times(workloads.config(0, requests=200), times)
    sim = mtsim.Simulator(w)
    sim.load()
    assert sim.run() == 0
    res, _, _ = sim.metrics()
    assert (res["finish_us"] > res["first_token_us"]).any()
    sim.close()
    assert np.isfinite(times).all()
