"""Infinities and NaN in tokens that a row does not see: the row is as if they
were not there, to the bit, wherever the tiles of keys end."""

import pytest

torch = pytest.importorskip("torch")
from paper_2608_16336_gb300 import instance_ops as ops  # noqa: E402
from test_instance_ops_gpu import BF, HF, device, prefill_case  # noqa: E402, F401

pytestmark = pytest.mark.gpu
JUNK = [float("nan"), float("inf"), float("-inf")]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("nq,nk,heads,value_dim", [
    ([200], [200], 2, 128), ([64, 100], [64, 100], 3, 72), ([300, 5], [301, 77], 2, 64),  # short prompts
    ([1000], [1000], 80, 128), ([700, 513], [900, 2600], 40, 104),                         # two tiles a block
    ([257], [5000], 1, 128), ([513, 300], [1300, 3001], 3, 40), ([700, 0], [600, 5000], 2, 8)])  # keys shared by blocks
def test_prefill_later_values_do_not_count(nq, nk, heads, value_dim, dtype):
    q, key, shared, value, qo, ko = prefill_case(nq, nk, heads, 128, 64, value_dim, dtype, seed=sum(nk))
    want, lse = ops.latent_prefill(q, key, shared, value, qo, ko, scale=0.1, longest=max(nq))
    junk = value.clone()
    first = {}  # the first query row of each request that sees each of the bad values
    for b, (a, n) in enumerate(zip(nq, nk)):
        for i, back in enumerate((1, 2, 3, 50, 130, 131, 190, 256)):
            j = n - back
            if j < 0 or a == 0:
                continue
            e = (7 * i + b) % value_dim
            junk[int(ko[b]) + j, i % heads, e] = JUNK[i % 3]
            first[b, i % heads, e, i] = (max(j - (n - a), 0), JUNK[i % 3])
    out, lse2 = ops.latent_prefill(q, key, shared, junk, qo, ko, scale=0.1, longest=max(nq))
    assert torch.equal(lse2, lse)
    hit = {}
    for (b, h, e, _), (row, x) in first.items():
        for r in range(row, nq[b]):
            hit.setdefault((int(qo[b]) + r, h, e), []).append(x)
    same = torch.ones_like(out, dtype=torch.bool)
    for at, xs in hit.items():
        same[at] = False
    assert torch.equal(out[same], want[same])
    at = torch.tensor(list(hit), device="cuda")
    expect = torch.tensor([sum(xs) for xs in hit.values()], device="cuda")
    assert torch.equal(torch.nan_to_num(out[at[:, 0], at[:, 1], at[:, 2]].float(), nan=0.5), torch.nan_to_num(expect, nan=0.5))
    again, _ = ops.latent_prefill(q, key, shared, junk, qo, ko, scale=0.1, longest=max(nq))
    assert torch.equal(torch.nan_to_num(again), torch.nan_to_num(out))
