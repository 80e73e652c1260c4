"""Rows of logits that verification of drafted tokens has to sum with care."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_verify_gpu import BF, F32, HF, check  # noqa: E402

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
