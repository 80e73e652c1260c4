"""The workspace's size is kept only when the library gave one (a fake library, no GPU)."""
import pytest

from paper_2608_16336_gb300 import mtsim

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402


class Library:
    def __init__(self, sizes):
        self.sizes, self.calls = list(sizes), 0

    def sim_op_latent_decode_workspace(self, *a):
        return self.sizes.pop(0)

    def sim_op_latent_decode(self, *a):
        self.calls += 1
        return 0

    def sim_op_last_error(self):
        return b"device query: not now"


def test_a_failed_size_is_not_kept(monkeypatch):
    fake = Library([0, 4096])
    monkeypatch.setattr(ops, "_LIB", fake)
    monkeypatch.setattr(ops, "_WORKSPACE", {})
    monkeypatch.setattr(ops, "_place", lambda *t: 0)
    monkeypatch.setattr(ops, "_stream_of", lambda device: 0)
    taken = []
    monkeypatch.setattr(ops, "_scratch", lambda nbytes, stream: taken.append(nbytes) or 256)
    monkeypatch.setattr(ops, "_release", lambda work: None)
    args = (torch.zeros(1, 1, 4, 576, dtype=torch.bfloat16), torch.zeros(2, 16, 576, dtype=torch.bfloat16),
            torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    with pytest.raises(mtsim.SimError, match="not now"):
        ops.latent_decode(*args, scale=1.0)
    assert not taken and not fake.calls
    for _ in range(2):
        ops.latent_decode(*args, scale=1.0)
    assert taken == [4096, 4096] and fake.calls == 2
