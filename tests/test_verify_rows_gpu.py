"""Rows of logits that verification of drafted tokens has to sum with care."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_verify_gpu import BF, F32, HF, check, gen  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    yield
    assert ops.faults() == 0


# the type's lowest number, the next ones, and others that a mask of lowest values or a large offset leaves
LEVELS = {HF: (-65504.0, -65472.0, -65376.0, -65000.0, -60000.0, -50000.0, -30000.0),
          BF: (torch.finfo(BF).min, -1e30, -9.95e29, -1e29, -65504.0, -60000.0),
          F32: (torch.finfo(F32).min, -1e30, -9.999999e29, -1e29, -65504.0, -60000.0)}


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("known", [True, False])
@pytest.mark.parametrize("t", [0.5, 1.0, 10.0, 100.0, 1000.0])
@pytest.mark.parametrize("vocab", [7, 8, 1001, 20003])
def test_rows_whose_largest_logit_is_near_the_lowest_number(vocab, t, known, dtype):
    """-infinity and NaN have no weight beside it, in the row or in the vectors that its ends share with others."""
    lowest, step = torch.finfo(dtype).min, max(1, vocab // 5)
    for none in (-math.inf, math.nan):
        b = len(LEVELS[dtype])
        target = torch.full((b, 2, vocab), none, device="cuda")
        for r, level in enumerate(LEVELS[dtype]):
            target[r, 0, r % vocab] = level  # one token
            target[r, 1, ::step] = level     # several, and one of the lowest number beside them
            target[r, 1, 1] = lowest
        target = target.to(dtype)
        tokens = torch.arange(b, device="cuda")[:, None] % vocab
        draft = target[:, 1:].contiguous() if known else None
        temperature = torch.full((b,), t, device="cuda")
        for u in (0.0, 0.9):
            uniform = torch.full((b, 2), u, device="cuda")
            check(target, tokens, uniform, draft, temperature, None, *ops.verify(target, tokens, uniform, draft=draft, temperature=temperature))


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("vocab", [1023, 4097, 20001, 131075])
@pytest.mark.parametrize("spread", [0.5, 3.0])
def test_equal_rows_leave_nothing_wherever_they_lie(spread, vocab, dtype):
    """Where target and draft are the same the next token comes from the target, as where the draft's row is empty (a
    call without drafts' rows cuts the target's into other chunks, whose sums differ in their last bits):
    rows off one another's place in a vector of 16 bytes are summed in other groups."""
    b, g = 60, gen(vocab)
    target = (torch.randn(b, 2, vocab, generator=g, device="cuda") * spread).to(dtype)
    tokens = torch.full((b, 1), -1, device="cuda")  # (refused)
    uniform = torch.rand(b, 2, generator=g, device="cuda")
    store = torch.zeros(b, vocab + 11, device="cuda", dtype=dtype)
    want = ops.verify(target, tokens, uniform, draft=torch.full_like(target[:, 1:], -math.inf))
    for first in (0, 1, 3, 8):
        draft = store[:, None, first:first + vocab]
        draft.copy_(target[:, :1])
        got = ops.verify(target, tokens, uniform, draft=draft)
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        check(target, tokens, uniform, draft, None, None, *got)
