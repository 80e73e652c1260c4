"""The count of waits that ran out is read when everything queued has ended."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402

pytestmark = pytest.mark.gpu


def test_faults_waits_for_every_stream():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    assert ops.faults() == 0
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)  # a tenth of a second
        done.record()
    assert not done.query()
    assert ops.faults() == 0
    assert done.query()
