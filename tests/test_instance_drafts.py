"""Drafted tokens of an instance: requests that have none, or fewer than others."""
import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_blocks import make, tokens, whole  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quantized", [False, True])
@pytest.mark.parametrize("drafts,counts", [([[-1], [-1], [4000]], [1, 1, 1]), ([[5, -1, 7], [-1, 5, 6], [9, 8, 2 ** 40]], [2, 1, 3])])
def test_where_a_request_has_no_draft_the_token_comes_from_the_target(drafts, counts, quantized):
    """Whatever the draft's logits hold in that place: as without them."""
    drafts = torch.tensor(drafts, device="cuda" if torch.cuda.is_available() else "cpu")
    new = drafts.shape[1] + 1
    for u in (0.1, 0.35, 0.8):
        got = []
        for known in (False, True):
            node = make(quantized)
            node.iterate([tokens(n, n) for n in (20, 31, 100)], uniform=torch.full((3,), 0.4, device="cuda"))
            draft = None
            if known:  # likely where the target's tokens are unlikely, and the other way round
                draft = torch.zeros(3, new - 1, 4000, device="cuda", dtype=torch.bfloat16)
                draft[..., 2000:] = -8.0
            uniform = torch.zeros(3, new, device="cuda")
            uniform[:, new - 1] = u
            _, t, kept, lp = node.speculate(drafts, draft=draft, uniform=uniform)
            whole(node, 120)
            got.append((t, lp))
            assert kept == counts
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert ops.faults() == 0
